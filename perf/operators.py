"""Performance cases of the stand-alone operators: the paged cache in 4 bits (plan, append, read, attend) and the log
probabilities of given tokens.

A case is one call (or the calls that belong together) on tensors that a serving program has in hand.  With `own` false
the same results are computed with elementary torch operations in 32 bits; exact() computes them in 64 bits.

The cache: a pool of blocks of block_tokens rows.  A block holds, per key head, the 4-bit codes of its keys
[block_tokens][head_dim / 2], those of its values, then a scale byte per 32 dims of every key and of every value.  A code is
sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6 (low half of a byte first), scale byte b stands for 2^(b - 127).
"""
import math
from types import SimpleNamespace

import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one verify pass of 48 conversations, 6 rows each: tables and slots of the rows, and the rejected ones given back
        dict(op="plan", name="plan_verify_48", seqs=48, block=64, lens_lo=600, lens_hi=9000, add_lo=6, add_hi=6),
        # prompts of 400 requests at once, one token to 700
        dict(op="plan", name="plan_prompts_400", seqs=400, block=16, lens_lo=0, lens_hi=64, add_lo=1, add_hi=700),
        # rows of a verify pass: 4 sequences x 8 rows, 40 key heads of 128, as fp32 activations
        dict(op="append", name="append_verify_32", rows=32, heads=40, hd=128, block=64, dtype="f32"),
        # a batch of prompts, 8 key heads, and the rows read back
        dict(op="append", name="append_prompts_9001", rows=9001, heads=8, hd=128, block=64, dtype="bf16"),
        # one drafted token of one short conversation: latency
        dict(op="attend", name="attend_token_650", seqs=1, rows_lo=1, rows_hi=1, past_lo=649, past_hi=649, heads=32, group=1, hd=128, block=64, dtype="bf16", tree=False),
        # a verify pass of four sequences, eight rows each, 13B widths
        dict(op="attend", name="attend_verify_4x8", seqs=4, rows_lo=8, rows_hi=8, past_lo=832, past_hi=1336, heads=40, group=1, hd=128, block=64, dtype="f32", tree=False),
        # a draft tree of 60 candidates and its root behind a long visual prompt, grouped heads
        dict(op="attend", name="attend_tree_61", seqs=1, rows_lo=61, rows_hi=61, past_lo=3014, past_hi=3014, heads=4, group=7, hd=128, block=64, dtype="f32", tree=True),
        # decode of 48 conversations of very different lengths, grouped heads
        dict(op="attend", name="attend_batch_48", seqs=48, rows_lo=1, rows_hi=1, past_lo=30, past_hi=16000, heads=8, group=8, hd=128, block=32, dtype="bf16", tree=False),
        # whole prompts, some of them behind a cached prefix
        dict(op="attend", name="attend_prompts_4", seqs=4, rows_lo=641, rows_hi=3008, past_lo=0, past_hi=1500, heads=8, group=4, hd=128, block=64, dtype="bf16", tree=False),
        # log probabilities of a verify pass's rows: the emitted token, five alternatives
        dict(op="logprobs", name="logprobs_verify_6", rows=6, vocab=32000, tokens=1, top=5, dtype="f32", temperature=1.0),
        # a serving batch with the widest vocabulary
        dict(op="logprobs", name="logprobs_batch_128", rows=128, vocab=152064, tokens=4, top=20, dtype="f32", temperature=0.7),
        # a prompt's own log probabilities
        dict(op="logprobs", name="logprobs_prompt_2040", rows=2040, vocab=32000, tokens=1, top=0, dtype="bf16", temperature=1.0),
    ]


def _spread(n, lo, hi):
    """n sizes spread over lo..hi on a logarithmic scale, in no order."""
    return [int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** (((i * 29) % n) / max(1, n - 1)))) - 1 for i in range(n)]


def _sizes(case):
    """rows of the call and cached rows (with those) of every sequence"""
    rows = _spread(case["seqs"], case["rows_lo"], case["rows_hi"])
    return rows, [r + p for r, p in zip(rows, reversed(_spread(case["seqs"], case["past_lo"], case["past_hi"])))]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("plan", "append", "attend", "attend", "attend", "logprobs"))
    if op == "plan":
        lo, add = rng.choice((0, 1, 300)), _log_int(rng, 1, 500)
        return dict(op=op, seqs=_log_int(rng, 1, 400), block=rng.choice((16, 32, 64, 128, 256)), lens_lo=lo, lens_hi=lo + _log_int(rng, 1, 8000), add_lo=min(add, rng.randint(0, 8)), add_hi=add)
    if op == "append":
        heads, hd = rng.choice((1, 4, 8, 32, 40)), rng.choice((64, 128))
        return dict(op=op, rows=_log_int(rng, 1, 9001 * 8 * 128 // (heads * hd)), heads=heads, hd=hd, block=rng.choice((16, 32, 64, 128)), dtype=rng.choice(("f32", "bf16")))
    if op == "logprobs":
        vocab = _log_int(rng, 1000, 152064)
        rows = _log_int(rng, 1, min(2040, 128 * 152064 // vocab))
        top = rng.choice((0, 1, 5, 20)) if rows <= 256 else 0
        return dict(op=op, rows=rows, vocab=vocab, tokens=rng.randint(1, 4), top=top, dtype=rng.choice(("f32", "bf16")), temperature=rng.choice((1.0, 0.7, 1.5)))
    heads, group = rng.choice(((4, 7), (32, 1), (40, 1), (8, 4), (8, 8), (4, 1), (1, 8), (2, 2)))
    hd, dtype, kind = rng.choice((64, 128)), rng.choice(("f32", "bf16")), rng.choice(("step", "step", "tree", "prompt"))
    case = dict(op=op, heads=heads, group=group, hd=hd, block=rng.choice((16, 32, 64, 128)), dtype=dtype, tree=kind == "tree")
    if kind == "prompt":
        lo = _log_int(rng, 100, 1000)
        return dict(case, seqs=rng.randint(1, 4), rows_lo=lo, rows_hi=lo + _log_int(rng, 1, 1000), past_lo=0, past_hi=rng.choice((0, rng.randint(1, 1500))))
    n = 1 if kind == "tree" else _log_int(rng, 1, 48)
    lo = rng.randint(2, 64) if kind == "tree" else rng.choice((1, 1, 5, 8))
    room = 48 * 1900 * 8 * 128 // (heads * hd)                # cached rows of all sequences together
    past = _log_int(rng, 1, max(2, min(16000, room // n)))
    return dict(case, seqs=n, rows_lo=lo, rows_hi=lo if kind == "tree" else max(lo, rng.choice((1, 6))), past_lo=rng.randint(0, past), past_hi=past)


# ---- inputs ---------------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"plan": _prepare_plan, "append": _prepare_append, "attend": _prepare_attend, "logprobs": _prepare_logprobs}[case["op"]](case, gen)


def _randint(gen, lo, hi, n):
    """n integers of lo..hi"""
    return torch.randint(lo, hi + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)


def _chunk(hd, block):
    return block * (hd + hd // 16)


def _prepare_plan(case, gen):
    n, T = case["seqs"], case["block"]
    keep = _randint(gen, case["lens_lo"], case["lens_hi"], n)
    add = _randint(gen, case["add_lo"], case["add_hi"], n)
    max_blocks = (case["lens_hi"] + case["add_hi"] + T - 1) // T
    n_blocks = n * max_blocks
    perm = torch.randperm(n_blocks, generator=gen, device="cuda").to(torch.int32)
    held = (keep + T - 1) // T
    start = held.cumsum(0) - held
    j = torch.arange(max_blocks, device="cuda")
    index = (start[:, None] + j).clamp(max=n_blocks - 1)
    table = torch.where(j < held[:, None], perm[index.long()], torch.full_like(index, -1).to(torch.int32)).to(torch.int32).contiguous()
    used = int(held.sum())
    free = torch.full((1 + n_blocks,), -1, dtype=torch.int32, device="cuda")
    free[0] = n_blocks - used
    free[1:1 + n_blocks - used] = perm[used:]
    rows = n * case["add_hi"]
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
    return SimpleNamespace(case=case, keep=keep, add=add, none=torch.zeros_like(add), held=held.to(torch.int32).contiguous(), table=table, free=free, n_blocks=n_blocks,
                           row_start=i32(n + 1), slots=i32(rows), positions=i32(rows), status=i32(n))


def _prepare_append(case, gen):
    rows, T, dt = case["rows"], case["block"], TYPES[case["dtype"]]
    n_blocks = (rows + T - 1) // T + 2
    slots = torch.randperm(n_blocks, generator=gen, device="cuda")[:(rows + T - 1) // T]
    slots = (slots[:, None] * T + torch.arange(T, device="cuda")).reshape(-1)[:rows].to(torch.int32).contiguous()
    shape = (rows, case["heads"], case["hd"])
    spread = torch.exp(0.7 * torch.randn(case["heads"], case["hd"], generator=gen, device="cuda"))       # channels of a key differ in size
    k = (torch.randn(shape, generator=gen, device="cuda") * spread).to(dt)
    v = torch.randn(shape, generator=gen, device="cuda").to(dt)
    pool = torch.zeros(n_blocks * case["heads"] * _chunk(case["hd"], T), dtype=torch.uint8, device="cuda")
    return SimpleNamespace(case=case, slots=slots, k=k, v=v, pool=pool, n_blocks=n_blocks, k_out=torch.empty_like(k), v_out=torch.empty_like(v))


def _prepare_attend(case, gen):
    heads, hd, T, dt = case["heads"], case["hd"], case["block"], TYPES[case["dtype"]]
    rows, lens = _sizes(case)
    n, total, hq = len(lens), sum(rows), heads * case["group"]
    nblk = [(x + T - 1) // T for x in lens]
    max_blocks, n_blocks = max(nblk), sum(nblk) + 1
    perm = torch.randperm(n_blocks, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((n, max_blocks), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, b in enumerate(nblk):
        table[s, :b] = perm[at:at + b]
        at += b
    chunk = _chunk(hd, T)
    pool = torch.empty((n_blocks, heads, chunk), dtype=torch.uint8, device="cuda")
    spread = torch.exp(0.5 * torch.randn(heads, 1, hd, generator=gen, device="cuda"))
    for b0 in range(0, n_blocks, 1024):
        b1 = min(n_blocks, b0 + 1024)
        k = torch.randn((b1 - b0, heads, T, hd), generator=gen, device="cuda") * spread
        v = torch.randn((b1 - b0, heads, T, hd), generator=gen, device="cuda")
        kc, ks = _codes(k)
        vc, vs = _codes(v)
        pool[b0:b1] = torch.cat([x.reshape(b1 - b0, heads, -1) for x in (kc, vc, ks, vs)], dim=-1)
    q = (torch.randn((total, hq, hd), generator=gen, device="cuda") / math.sqrt(float(spread.square().mean()))).to(dt)
    mask = None
    if case["tree"]:                                   # rows of a draft tree: row i sees itself and the rows its parent sees
        pick = torch.rand(total, generator=gen, device="cuda").tolist()
        bits, at = [], 0
        for r in rows:
            own_bits = []
            for i in range(r):
                own_bits.append((own_bits[int(pick[at + i] * i)] if i else 0) | 1 << i)
            bits += own_bits
            at += r
        mask = torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64, device="cuda")
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    s = SimpleNamespace(case=case, rows=rows, lens=lens, pool=pool.reshape(-1), n_blocks=n_blocks, table=table, q=q, mask=mask, out=torch.empty_like(q), workspace=None,
                        row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2509_23928_amd as hv
        s.shape = hv.Kv4Shape(heads, hd, T, n_blocks)
        s.workspace = torch.zeros(hv.kv4_attend_bytes(s.shape, hq, n, max(rows), max(lens), dt), dtype=torch.uint8, device="cuda")
    return s


def _codes(x):
    """codes (two to a byte) and scale bytes of x, groups of 32 along the last dim"""
    g = x.unflatten(-1, (-1, 32))
    a = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(a)                               # a = m 2^e, m in [0.5, 1)
    e = torch.where(m * 2 <= 1.75, e - 3, e - 2).clamp(-100, 125)
    y = torch.ldexp(g.abs(), -e)
    code = torch.zeros_like(y, dtype=torch.uint8)
    for border, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):       # a value on a border: the even code
        code += (y >= border) if up else (y > border)
    code += (g < 0).to(torch.uint8) * 8
    pair = code.flatten(-2).unflatten(-1, (-1, 2))
    return pair[..., 0] | pair[..., 1] << 4, (e + 127).squeeze(-1).to(torch.uint8)


def _prepare_logprobs(case, gen):
    rows, vocab, dt = case["rows"], case["vocab"], TYPES[case["dtype"]]
    x = torch.randn((rows, vocab), generator=gen, device="cuda") * 2.5
    x[:, :: max(1, vocab // 40)] += 6.0 * torch.rand((rows, len(range(0, vocab, max(1, vocab // 40)))), generator=gen, device="cuda")      # a few tokens stand out
    x = x.to(dt)
    tokens = _randint(gen, 0, vocab - 1, rows * case["tokens"]).reshape(rows, -1)
    tokens[:, 0] = x.argmax(-1).to(torch.int32)
    s = SimpleNamespace(case=case, logits=x, tokens=tokens.contiguous(), workspace=None)
    f32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device="cuda")
    s.logprob, s.entropy = f32(rows, case["tokens"]), f32(rows)
    s.top_ids = torch.empty((rows, case["top"]), dtype=torch.int32, device="cuda") if case["top"] else None
    s.top_logprobs = f32(rows, case["top"]) if case["top"] else None
    if own:
        import paper_2509_23928_amd as hv
        s.workspace = torch.zeros(hv.logprobs_bytes(rows, vocab, case["top"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------------

def run(state):
    return globals()[("_own_" if own else "_plain_") + state.case["op"]](state)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _own_plan(s):
    import paper_2509_23928_amd as hv
    for add in (s.none, s.add):                         # the rows of the pass before are given back, then the next pass's are planned
        hv.kv4_plan(s.keep, add, s.held, s.table, s.free, s.row_start, s.slots, s.positions, s.status, block_tokens=s.case["block"], n_blocks=s.n_blocks, stream=_stream())
    return s.held, s.table, s.free, s.row_start, s.slots, s.positions, s.status


def _own_append(s):
    import paper_2509_23928_amd as hv
    c = s.case
    shape = hv.Kv4Shape(c["heads"], c["hd"], c["block"], s.n_blocks)
    hv.kv4_append(shape, s.pool, s.slots, s.k, s.v, stream=_stream())
    hv.kv4_read(shape, s.pool, s.slots, s.k_out, s.v_out, stream=_stream())
    return s.k_out, s.v_out


def _own_attend(s):
    import paper_2509_23928_amd as hv
    hv.kv4_attend(s.shape, s.pool, s.table, s.row_start, s.kv_len, s.q, s.out, max_rows=max(s.rows), max_len=max(s.lens), workspace=s.workspace,
                  mask=s.mask, stream=_stream())
    return s.out


def _own_logprobs(s):
    import paper_2509_23928_amd as hv
    hv.logprobs(s.logits, s.tokens, s.logprob, s.entropy, s.top_ids, s.top_logprobs, temperature=s.case["temperature"], workspace=s.workspace, stream=_stream())
    return tuple(t for t in (s.logprob, s.entropy, s.top_ids, s.top_logprobs) if t is not None)


def _plain_plan(s):
    _plain_plan_once(s, s.none)
    _plain_plan_once(s, s.add)
    return s.held, s.table, s.free, s.row_start, s.slots, s.positions, s.status


def _plain_plan_once(s, add):
    T, keep, held, table, free = s.case["block"], s.keep, s.held, s.table, s.free
    n, max_blocks = table.shape
    need = (keep + add + T - 1) // T
    valid = (keep >= 0) & (add >= 0) & (keep <= held * T) & (need <= max_blocks)
    fits = add.where(valid, 0).cumsum(0) <= s.slots.numel()
    good = valid & fits
    j = torch.arange(max_blocks, device="cuda")
    # blocks given back: the last sequence's last block first
    gone = (good[:, None] & (j >= need[:, None]) & (j < held[:, None])).flip((0, 1)).reshape(-1)
    at = torch.where(gone, free[0] + gone.cumsum(0), free.numel())
    free = torch.cat((free, free[:1])).scatter(0, at.long(), table.flip((0, 1)).reshape(-1))[:-1]
    table = table.masked_fill(gone.reshape(n, max_blocks).flip((0, 1)), -1)
    count = free[0] + gone.sum()
    # blocks taken, from the top of the list, in order of the sequences
    grow = (need - held).clamp(min=0).where(good, 0)
    upto = grow.cumsum(0)
    served = good & ((grow == 0) | (upto <= count))
    taken = served[:, None] & (j >= held[:, None]) & (j < need[:, None])
    source = count - (upto - grow)[:, None] - (j - held[:, None])
    table = torch.where(taken, free[source.clamp(1, free.numel() - 1).long()], table)
    free[0] = count - grow.where(served, 0).sum()
    s.held, s.table, s.free = torch.where(served, need, held).to(torch.int32), table, free
    s.status = torch.where(~valid, 2, torch.where(~fits, 3, torch.where(served, 0, 1))).to(torch.int32)
    ends = add.where(served, 0).cumsum(0)
    s.row_start = torch.cat((ends.new_zeros(1), ends)).to(torch.int32)
    r = torch.arange(s.slots.numel(), device="cuda")
    seq = torch.searchsorted(ends, r, right=True).clamp(max=n - 1)
    pos = keep[seq] + r - s.row_start[seq]
    inside = r < ends[-1]
    s.slots = torch.where(inside, table[seq, (pos // T).clamp(0, max_blocks - 1)] * T + pos % T, -1).to(torch.int32)
    s.positions = torch.where(inside, pos, -1).to(torch.int32)


def _plain_append(s):
    c = s.case
    hd, T = c["hd"], c["block"]
    block, row = (s.slots // T).long(), (s.slots % T).long()
    pool = s.pool.view(s.n_blocks, c["heads"], -1)
    h = torch.arange(c["heads"], device="cuda")[None, :, None]
    outs, at = [], 0
    for x in (s.k, s.v):
        code, scale = _codes(x.float())
        for part, base, width in ((code, at * T * hd // 2, hd // 2), (scale, T * hd + at * T * hd // 32, hd // 32)):
            pool[block[:, None, None], h, base + row[:, None, None] * width + torch.arange(width, device="cuda")] = part
        at += 1
    for i, like in enumerate((s.k, s.v)):
        parts = []
        for base, width in ((i * T * hd // 2, hd // 2), (T * hd + i * T * hd // 32, hd // 32)):
            parts.append(pool[block[:, None, None], h, base + row[:, None, None] * width + torch.arange(width, device="cuda")])
        outs.append(_values(*parts).to(like.dtype))
    return tuple(outs)


def _values(code, scale):
    """fp32 values of codes [..., w / 2] with scale bytes [..., w / 32]"""
    lut = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float32, device=code.device)
    x = lut[torch.stack((code & 15, code >> 4), -1).flatten(-2).long()]
    size = (scale.to(torch.int32) << 23).view(torch.float32)
    size = torch.where(scale == 255, float("nan"), size)
    return (x.unflatten(-1, (-1, 32)) * size[..., None]).flatten(-2)


def _cached(s, seq):
    """keys and values of one sequence, [heads][rows][hd]"""
    c = s.case
    hd, T, length = c["hd"], c["block"], s.lens[seq]
    nb = (length + T - 1) // T
    chunk = s.pool.view(s.n_blocks, c["heads"], -1)[s.table[seq, :nb].long()].transpose(0, 1)
    cut = (0, T * hd // 2, T * hd, T * hd + T * hd // 32, T * (hd + hd // 16))
    kc, vc, ks, vs = (chunk[:, :, a:b].reshape(c["heads"], nb * T, -1)[:, :length] for a, b in zip(cut, cut[1:]))
    return kc, ks, vc, vs


def _seen(s, seq, first):
    """which keys each row of a sequence sees, [rows][keys]"""
    rows, length = s.rows[seq], s.lens[seq]
    i, j = torch.arange(rows, device="cuda")[:, None], torch.arange(length, device="cuda")[None]
    new = j - (length - rows)
    if s.mask is None:
        return new <= i
    return (new < 0) | ((s.mask[first:first + rows, None] >> new.clamp(min=0)) & 1).bool()


def _plain_attend(s):
    c, first, outs = s.case, 0, []
    heads, group, hd = c["heads"], c["group"], c["hd"]
    for seq, rows in enumerate(s.rows):
        kc, ks, vc, vs = _cached(s, seq)
        k, v = _values(kc, ks), _values(vc, vs)
        q = s.q[first:first + rows].float().view(rows, heads, group, hd).permute(1, 2, 0, 3).reshape(heads, group * rows, hd)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) * (hd ** -0.5)
        x = x.view(heads, group, rows, -1).masked_fill(~_seen(s, seq, first), -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        o = torch.matmul(p.view(heads, group * rows, -1), v).view(heads, group, rows, hd) / p.sum(-1, keepdim=True)
        outs.append(o.permute(2, 0, 1, 3).reshape(rows, heads * group, hd).to(s.q.dtype))
        first += rows
    return torch.cat(outs)


def _plain_logprobs(s):
    x = s.logits.float() / s.case["temperature"]
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    z = e.sum(-1, keepdim=True)
    log_z = torch.log(z)
    entropy = (log_z - (e * (x - top)).sum(-1, keepdim=True) / z).squeeze(-1)
    given = x.gather(-1, s.tokens.long()) - top - log_z
    if not s.case["top"]:
        return given, entropy
    value, index = torch.sort(s.logits, dim=-1, descending=True, stable=True)
    index = index[:, :s.case["top"]]
    return given, entropy, index.to(torch.int32), x.gather(-1, index) - top - log_z


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "plan":
        n, T = case["seqs"], case["block"]
        add = (case["add_lo"] + case["add_hi"]) / 2
        # both calls: lengths in, starts, status and held blocks out; the second one's slots and positions; blocks moved twice, table and list
        return dict(bytes=int(2 * 20 * n + 8 * n * case["add_hi"] + 2 * 8 * n * add / T), flops=0)
    if op == "append":
        values = 2 * case["rows"] * case["heads"] * case["hd"]
        size = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=int(values * (2 * size + 2 * 17 / 32) + 8 * case["rows"]), flops=0)        # in, cache out, cache in, out
    if op == "attend":
        hq, hd = case["heads"] * case["group"], case["hd"]
        size = 4 if case["dtype"] == "f32" else 2
        rows, lens = _sizes(case)
        pairs = sum(r * (n - r) + (6 * r if case["tree"] else r * (r + 1) // 2) for r, n in zip(rows, lens))
        return dict(bytes=2 * sum(rows) * hq * hd * size + sum(lens) * case["heads"] * (hd + hd // 16) + 4 * sum((n + case["block"] - 1) // case["block"] + 2 for n in lens),
                    flops=4 * pairs * hq * hd)
    size = 4 if case["dtype"] == "f32" else 2
    return dict(bytes=case["rows"] * (case["vocab"] * size + 8 * case["tokens"] + 4 + 8 * case["top"]), flops=4 * case["rows"] * case["vocab"])


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------------

def exact(case, seed):
    op = case["op"]
    if op == "plan":
        return None                                     # whole numbers: the plain form has them
    s = prepare(case, seed)
    if op == "append":
        return tuple(_exact_rounded(x) for x in (s.k, s.v))
    if op == "logprobs":
        x = s.logits.double() / case["temperature"]
        log_p = torch.log_softmax(x, -1)
        entropy = -(log_p.exp() * log_p).sum(-1)
        given = torch.gather(log_p, 1, s.tokens.long())
        if not case["top"]:
            return given, entropy
        # the value falls, then the index rises
        order = torch.sort(-s.logits.double(), dim=-1, stable=True).indices[:, :case["top"]]
        return given, entropy, order.to(torch.int32), torch.gather(log_p, 1, order)
    out = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")
    first = 0
    for seq, (rows, length) in enumerate(zip(s.rows, s.lens)):
        kc, ks, vc, vs = _cached(s, seq)
        see = _seen(s, seq, first)
        for h in range(case["heads"]):
            k, v = _exact_values(kc[h], ks[h]), _exact_values(vc[h], vs[h])
            for g in range(case["group"]):
                hq = h * case["group"] + g
                x = (s.q[first:first + rows, hq].double() @ k.T) / math.sqrt(case["hd"])
                out[first:first + rows, hq] = torch.softmax(x.masked_fill(~see, -math.inf), -1) @ v
        first += rows
    return out


def _exact_values(code, scale):
    half = torch.stack((code % 16, code // 16), -1).flatten(-2).to(torch.int64)
    e, m = (half % 8) // 2, half % 2                    # two bits of exponent, one of mantissa
    size = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e - 1).double())
    sign = 1 - 2 * (half // 8).double()
    return sign * size * torch.exp2(scale.double() - 127).repeat_interleave(32, -1)


def _exact_rounded(x):
    """x rounded to the format, from its definition: the nearest of the sixteen values at the group's scale"""
    g = x.double().unflatten(-1, (-1, 32))
    a = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(a.clamp(min=1e-300)))
    e = torch.where(a / 2.0 ** e > 1.75, e - 1, e - 2).clamp(-100, 125)
    y = (g / 2.0 ** e).abs()
    best, far = torch.zeros_like(y), torch.full_like(y, math.inf)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):                  # even codes first: a tie stays with them
        d = (y - LEVELS[i]).abs()
        best, far = torch.where(d < far, LEVELS[i], best), torch.minimum(d, far)
    return (torch.copysign(best, g) * 2.0 ** e).flatten(-2)
