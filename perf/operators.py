"""The operators of a paged K/V cache, as measurable cases.

Writing new K/V rows into a paged cache (quantising them as they are written where the cache
holds 8-bit floats with an exponent per position and head), reading entries back, and the
attention of a chunk of new tokens (one token to thousands, ragged over the sequences) that reads
such a cache.  Each operator in its plain form (elementary torch operations in 32 bits), as the
calls that a program makes of this framework, and in 64 bits from its definition.

The cache: K and V as [block][kv head][16 positions][head_dim], a table of blocks per sequence.
The 8-bit form: for each position and kv head, with a = max |x| = m 2^E, m in [1/2, 1), the
exponent e = E - 9 (E - 8 where m > 7/8; 0 for a = 0), and the codes e4m3(x 2^-e), so that the
largest element is at most 448 = 7/8 2^9; the stored byte is e + 127.
"""
import math

import torch

own = False

BT = 16   # positions per block
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # ---- attention of new tokens over the cache
        # one user of a small decoder (GPT-2-small's heads), next token: latency is all there is
        dict(name="attn_step_small", kind="attn", kv="bf16", heads=12, kv_heads=12, head_dim=64, new="1", past="332"),
        # the fp32 decoder of the tests, a short turn
        dict(name="attn_turn_f32", kind="attn", kv="f32", heads=4, kv_heads=4, head_dim=64, new="17,5", past="64,96"),
        # next tokens of 16 users of a grouped-query decoder, ragged contexts, 8-bit cache
        dict(name="attn_steps_gqa_e4m3", kind="attn", kv="e4m3", heads=32, kv_heads=8, head_dim=128, new="1,1,1,1,1,1,1,1,1,1,1,1,1,1,1,1",
             past="4095,117,2048,15,3001,640,999,1,2500,1777,64,3333,250,4000,31,1500"),
        # next token of one user far into a long context, 8-bit cache: a stream of K and V
        dict(name="attn_step_long_e4m3", kind="attn", kv="e4m3", heads=32, kv_heads=32, head_dim=128, new="1", past="30010"),
        # four users, five proposed tokens each to check at once, over the benchmark's 2048-token context
        dict(name="attn_check_bf16", kind="attn", kv="bf16", heads=32, kv_heads=32, head_dim=128, new="5,5,4,5",
             past="2048,2100,1990,2303"),
        # a user's next message: 256 tokens on a 4096-token conversation
        dict(name="attn_turn_bf16", kind="attn", kv="bf16", heads=32, kv_heads=32, head_dim=128, new="256", past="4096"),
        # a server's mixed batch: idle, generating, and reading users together, 8-bit cache
        dict(name="attn_mixed_e4m3", kind="attn", kv="e4m3", heads=32, kv_heads=8, head_dim=128,
             new="1,0,37,512,1,1,128,3", past="2047,500,0,1531,8000,77,4096,1200"),
        # a piece of a long document: 2048 tokens on 16384 before them
        dict(name="attn_document_bf16", kind="attn", kv="bf16", heads=32, kv_heads=8, head_dim=128, new="2048", past="16384"),
        # ---- quantised as written, and read back
        # the K/V of a step's 8 tokens, written and read back
        dict(name="store_step", kind="store", src="bf16", kv_heads=32, head_dim=128, rows=8, seqs=8, pad=0),
        # the K/V of a prompt's tokens out of a product that also holds Q, some rows padding
        dict(name="store_prompt", kind="store", src="bf16", kv_heads=32, head_dim=128, rows=2048, seqs=1, pad=37),
        # a small fp32 source with heads of 64, several sequences
        dict(name="store_f32", kind="store", src="f32", kv_heads=12, head_dim=64, rows=777, seqs=5, pad=0),
        # a whole conversation read back in bf16
        dict(name="read_conversation", kind="read", dst="bf16", kv_heads=32, head_dim=128, rows=30011, seqs=3),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    text = lambda ns: ",".join(str(n) for n in ns)  # noqa: E731
    kind = rng.choice(["step", "step", "check", "turn", "turn", "mixed", "f32", "store", "store", "read"])
    heads, kv_heads, dh = rng.choice([(12, 12, 64), (32, 32, 128), (32, 8, 128), (16, 2, 64), (4, 2, 128), (25, 25, 64)])
    kv = rng.choice(["bf16", "e4m3"])
    if kind == "step":
        n = _log_int(rng, 1, 64)
        return dict(kind="attn", kv=kv, heads=heads, kv_heads=kv_heads, head_dim=dh, new=text([1] * n),
                    past=text(_log_int(rng, 1, 120000 // n) for _ in range(n)))
    if kind == "check":
        n = _log_int(rng, 1, 16)
        return dict(kind="attn", kv=kv, heads=heads, kv_heads=kv_heads, head_dim=dh,
                    new=text(rng.randint(2, 12) for _ in range(n)), past=text(_log_int(rng, 1, 60000 // n) for _ in range(n)))
    if kind == "turn":
        return dict(kind="attn", kv=kv, heads=heads, kv_heads=kv_heads, head_dim=dh, new=text([_log_int(rng, 13, 2048)]),
                    past=text([_log_int(rng, 1, 16000) - 1]))
    if kind == "mixed":
        n = rng.randint(2, 8)
        return dict(kind="attn", kv=kv, heads=heads, kv_heads=kv_heads, head_dim=dh,
                    new=text([rng.choice([0, 1, 1, _log_int(rng, 2, 512)]) for _ in range(n - 1)] + [_log_int(rng, 1, 512)]),
                    past=text(_log_int(rng, 1, 8000) - 1 for _ in range(n)))
    if kind == "f32":
        n = rng.randint(1, 4)
        heads, kv_heads, dh = rng.choice([(4, 4, 64), (4, 2, 32), (2, 1, 128)])
        return dict(kind="attn", kv="f32", heads=heads, kv_heads=kv_heads, head_dim=dh,
                    new=text(_log_int(rng, 1, 64) for _ in range(n)),
                    past=text(_log_int(rng, 1, 512) - 1 for _ in range(n)))
    seqs = rng.randint(1, 8)
    if kind == "store":
        rows = max(seqs, _log_int(rng, 1, 8192))
        return dict(kind="store", src=rng.choice(["bf16", "bf16", "f32"]), kv_heads=kv_heads, head_dim=dh, rows=rows,
                    seqs=seqs, pad=rng.choice([0, 0, rows // 9]))
    return dict(kind="read", dst=rng.choice(["bf16", "bf16", "f32"]), kv_heads=kv_heads, head_dim=dh,
                rows=max(seqs, _log_int(rng, 1, 40000)), seqs=seqs)


def _lens(case):
    """New tokens and cached positions before them, per sequence."""
    return tuple([int(n) for n in case[k].split(",")] for k in ("new", "past"))


def work(case):
    hk, dh = case["kv_heads"], case["head_dim"]
    if case["kind"] == "attn":
        kv_b = {"f32": 4 * dh, "bf16": 2 * dh, "e4m3": dh + 1}[case["kv"]]
        q_b = 4 if case["kv"] == "f32" else 2
        new, past = _lens(case)
        rows = sum(new)
        keys = sum(n + p for n, p in zip(new, past) if n)
        pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(new, past))
        return {"bytes": 2 * rows * case["heads"] * dh * q_b + 2 * keys * hk * kv_b,
                "flops": 4 * dh * case["heads"] * pairs}
    if case["kind"] == "store":
        b = 4 if case["src"] == "f32" else 2
        live = case["rows"] - case["pad"]
        # read, written in 8 bits, read back as the source's type
        return {"bytes": 2 * live * hk * (dh * b + 2 * (dh + 1) + dh * b), "flops": 0}
    b = 4 if case["dst"] == "f32" else 2
    return {"bytes": 2 * case["rows"] * hk * (dh + 1 + dh * b), "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 17)
    return g


def _table(seq_positions, g):
    """Blocks for each sequence's positions, in a shuffled order, and the table of them."""
    need = [max(1, (n + BT - 1) // BT) for n in seq_positions]
    total, width = sum(need) + 3, max(need)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(need), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, total


def _values(shape, g, spread):
    """K / V like values: normal, with channels and positions of different sizes."""
    x = torch.randn(shape, generator=g, device="cuda")
    ch = torch.exp2(spread * torch.randn(shape[-1], generator=g, device="cuda"))
    return x * ch


def _split(rows, seqs):
    """rows positions dealt out to seqs sequences, the first ones longer."""
    left, out = rows, []
    for s in range(seqs):
        n = left if s == seqs - 1 else max(1, min(left - (seqs - 1 - s), left * 2 // (seqs - s + 1)))
        out.append(n)
        left -= n
    return out


def _pow2(e):
    """2^e, -126 <= e <= 127, as float32: the exponent's bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _encode(x):
    """Codes (as float8) and stored exponents of rows x [..., head_dim], in 32 bits."""
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m == 0, torch.zeros_like(e), (e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-126))
    return (x * _pow2(-e).unsqueeze(-1)).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _cache_type(case):
    return case["kv"] if case["kind"] == "attn" else "e4m3"


def prepare(case, seed):
    g = _gen(seed)
    hk, dh = case["kv_heads"], case["head_dim"]
    st = {"case": case}
    if case["kind"] == "attn":
        h = case["heads"]
        new, past = _lens(case)
        lens = [n + p for n, p in zip(new, past)]
        table, blocks = _table(lens, g)
        dt = torch.float32 if case["kv"] == "f32" else torch.bfloat16
        k = _values((blocks, hk, BT, dh), g, 0.5).to(dt)
        v = _values((blocks, hk, BT, dh), g, 0.25).to(dt)
        rows = sum(new)
        # the queries as the first columns of a product that also holds the new K and V
        st["q"] = (1.2 * torch.randn(rows, h + 2 * hk, dh, generator=g, device="cuda")).to(dt)[:, :h]
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        st["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        st["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        st["max_q"], st["max_kv"] = max(new), max(lens)
    else:
        rows, seqs = case["rows"], case["seqs"]
        live = rows - case.get("pad", 0)
        per = _split(live, seqs)
        table, blocks = _table([n + 5 for n in per], g)
        seq = torch.cat([torch.full((n,), s, dtype=torch.int32) for s, n in enumerate(per)])
        pos = torch.cat([torch.arange(n, dtype=torch.int32) + 3 for n in per])
        if rows > live:   # padding rows stand behind the live ones
            seq = torch.cat([seq, torch.full((rows - live,), -1, dtype=torch.int32)])
            pos = torch.cat([pos, torch.zeros(rows - live, dtype=torch.int32)])
        st["seq"], st["pos"] = seq.cuda(), pos.cuda()
        st["live"] = live
        if case["kind"] == "store":
            x = _values((rows, 3 * hk, dh), g, 1.0).to(TYPES[case["src"]])
            st["k_new"], st["v_new"] = x[:, hk:2 * hk], x[:, 2 * hk:]
            k = v = torch.zeros(blocks, hk, BT, dh, device="cuda")
        else:
            k = _values((blocks, hk, BT, dh), g, 1.0)
            v = _values((blocks, hk, BT, dh), g, 1.0)
    if _cache_type(case) == "e4m3":
        (k, ke), (v, ve) = _encode(k.float()), _encode(v.float())
    else:
        ke = ve = None
    st.update(k=k, v=v, ke=ke, ve=ve, table=table)
    if own:
        import paper_2601_03700_gb300 as adept
        c = adept.KVCache(blocks, hk, dh, table.shape[0], table.shape[1], dtype=_cache_type(case), block_tokens=BT)
        c.block_table.copy_(table)
        c.k.copy_(k.view(c.k.dtype) if ke is not None else k)
        c.v.copy_(v.view(c.v.dtype) if ke is not None else v)
        if ke is not None:
            c.k_exp.copy_(ke)
            c.v_exp.copy_(ve)
        st["cache"] = c
        if case["kind"] == "attn":
            st["ws"] = c.attention_workspace(case["heads"], st["q"].shape[0], st["max_q"], st["max_kv"])
    return st


# ---------------------------------------------------------------------------
# the passes
# ---------------------------------------------------------------------------

def _decode(codes, exps):
    return codes.float() * _pow2(exps.int() - 127).unsqueeze(-1)


def _positions(st, pool, exps, s, n):
    """Positions 0..n-1 of sequence s out of a pool, in 32 bits, [kv head][position][head_dim]."""
    b = st["table"][s, :(n + BT - 1) // BT].long()
    x = pool[b].float() if exps is None else _decode(pool[b], exps[b])
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def _plain_attention(st):
    case = st["case"]
    q, dh, group = st["q"], case["head_dim"], case["heads"] // case["kv_heads"]
    out = torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    r = 0
    for s, (n, past) in enumerate(zip(*_lens(case))):
        if n == 0:
            continue
        k = _positions(st, st["k"], st["ke"], s, n + past)
        v = _positions(st, st["v"], st["ve"], s, n + past)
        # [kv head][new token x head of the group][dim]
        qs = q[r:r + n].float().view(n, case["kv_heads"], group, dh).permute(1, 0, 2, 3).reshape(case["kv_heads"], n * group, dh)
        sc = torch.matmul(qs, k.transpose(1, 2)) * (1.0 / math.sqrt(dh))
        if n > 1:
            at = torch.arange(n, device="cuda").repeat_interleave(group) + past
            late = torch.arange(n + past, device="cuda")[None, :] > at[:, None]
            sc.masked_fill_(late[None], float("-inf"))
        sc = torch.exp(sc - sc.amax(-1, keepdim=True))
        o = torch.matmul(sc, v) / sc.sum(-1, keepdim=True)
        out[r:r + n] = o.view(case["kv_heads"], n, group, dh).permute(1, 0, 2, 3).reshape(n, case["heads"], dh).to(q.dtype)
        r += n
    return out


def _plain_read(st, dtype, live):
    seq, pos = st["seq"][:live].long(), st["pos"][:live].long()
    b = st["table"][seq, pos // BT].long()
    return [_decode(st[a][b, :, pos % BT], st[a + "e"][b, :, pos % BT]).to(dtype) for a in ("k", "v")]


def _plain_store(st):
    live = st["live"]
    seq, pos = st["seq"][:live].long(), st["pos"][:live].long()
    b = st["table"][seq, pos // BT].long()
    for a in ("k", "v"):
        codes, exps = _encode(st[a + "_new"][:live].float())
        st[a][b, :, pos % BT] = codes
        st[a + "e"][b, :, pos % BT] = exps


def run(state):
    case = state["case"]
    if not own:
        if case["kind"] == "attn":
            return _plain_attention(state)
        if case["kind"] == "store":
            _plain_store(state)
            return _plain_read(state, TYPES[case["src"]], state["live"])
        return _plain_read(state, TYPES[case["dst"]], case["rows"])
    import paper_2601_03700_gb300 as adept
    c = state["cache"]
    if case["kind"] == "attn":
        q = state["q"]
        out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
        adept.adept_chunk_attention(c, q, state["q_start"], state["kv_len"], state["max_q"], state["max_kv"], out, state["ws"])
        return out
    if case["kind"] == "store":
        adept.adept_kv_append(c, state["k_new"], state["v_new"], state["seq"], state["pos"])
        dt, n = TYPES[case["src"]], state["live"]
    else:
        dt, n = TYPES[case["dst"]], case["rows"]
    k = torch.empty(n, case["kv_heads"], case["head_dim"], dtype=dt, device="cuda")
    v = torch.empty_like(k)
    adept.adept_kv_gather(c, state["seq"][:n], state["pos"][:n], k, v)
    return [k, v]


# ---------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _exact_quantised(x):
    """x rounded to the nearest value the 8-bit form holds (ties to the even code), in 64 bits."""
    x = x.double()
    a = x.abs().amax(-1, keepdim=True)
    # the smallest power of two (from 2^-126 on) that brings the row's largest value to 448 or below
    e = torch.ceil(torch.log2(torch.where(a > 0, a, torch.full_like(a, 448.0)) / 448.0))
    e = torch.where(a <= 448.0 * torch.exp2(e - 1), e - 1, e)   # log2 may be off by an ulp next to a power of two
    e = torch.where(a > 448.0 * torch.exp2(e), e + 1, e).clamp(min=-126)
    y = x / torch.exp2(e)
    # spacing of e4m3 at y: 2^(floor(log2 |y|) - 3), 2^-9 below 2^-6
    b = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    b = torch.where(torch.exp2(b + 1) <= y.abs(), b + 1, b)
    b = torch.where(torch.exp2(b) > y.abs(), b - 1, b).clamp(min=-6)
    step = torch.exp2(b - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def exact(case, seed):
    global own
    held, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = held
    if case["kind"] == "store":
        return [_exact_quantised(st[a][:st["live"]]) for a in ("k_new", "v_new")]
    if case["kind"] == "read":
        out = []
        for a in ("k", "v"):
            val = st[a].double() * torch.exp2(st[a + "e"].double() - 127).unsqueeze(-1)
            s, p = st["seq"].long(), st["pos"].long()
            out.append(val[st["table"].long()[s, p // BT], :, p % BT])
        return out
    h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.zeros(sum(_lens(case)[0]), h, dh, dtype=torch.float64, device="cuda")
    r = 0
    for s, (n, past) in enumerate(zip(*_lens(case))):
        total = n + past
        p = torch.arange(total, device="cuda")
        blk = st["table"].long()[s, p // BT]
        for kh in range(hk if n else 0):
            kk, vv = (st[a][blk, kh, p % BT].double() for a in ("k", "v"))
            if st["ke"] is not None:
                kk = kk * torch.exp2(st["ke"][blk, kh, p % BT].double() - 127)[:, None]
                vv = vv * torch.exp2(st["ve"][blk, kh, p % BT].double() - 127)[:, None]
            for head in range(kh * (h // hk), (kh + 1) * (h // hk)):
                w = (st["q"][r:r + n, head].double() @ kk.T) / math.sqrt(dh)
                w[p[None, :] > past + torch.arange(n, device="cuda")[:, None]] = -math.inf
                out[r:r + n, head] = torch.softmax(w, dim=-1) @ vv
        r += n
    return out
