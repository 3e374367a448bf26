"""The operators on callers' tensors on the GPU against their definitions in 64 bits (operator_reference.py)."""
import math
import random

import numpy as np
import pytest

import operator_reference as ref

torch = pytest.importorskip("torch")
import paper_2509_23928_amd as hv                                      # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"


def stream():
    return torch.cuda.current_stream().cuda_stream


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)


def f64(t):
    return t.detach().double().cpu().numpy()


# ---- append and read ---------------------------------------------------------------------------------------------------------------

def special_rows(rng, shape):
    """Rows with the values that decide a code: ties, the border of the scale, zeros, tiny and huge ones."""
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-3, 3, shape[:-1] + (1,)))
    flat = x.reshape(-1, 32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, -0.25, -0.75, -5.0])
    for i in range(0, len(flat), 5):
        flat[i, :12] = ties
        flat[i, 12:] *= 0.01
    for i in range(1, len(flat), 7):
        flat[i] = 0.0
    for i in range(2, len(flat), 11):
        flat[i] *= 2.0 ** -110
    for i in range(3, len(flat), 13):
        flat[i, 0], flat[i, 1:] = 1.75 * 2.0 ** 20, flat[i, 1:] / 8          # 7 / 4: the last one that the smaller scale takes
        flat[i + 1 if i + 1 < len(flat) else i, 0] = (1.75 + 2.0 ** -7) * 2.0 ** 20
    return x


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("heads,hd,block,rows,stride", [(1, 64, 16, 1, "plain"), (3, 128, 64, 33, "padded"), (4, 64, 32, 130, "heads first"), (8, 128, 256, 77, "plain"), (40, 128, 16, 9, "padded"), (2, 64, 32, 9001, "plain"),
                                                         (3, 128, 64, 4099, "padded")])
def test_append_and_read(dtype, heads, hd, block, rows, stride):
    rng = np.random.default_rng(rows * hd)
    dt = getattr(torch, dtype)
    x = [torch.as_tensor(special_rows(rng, (rows, heads, hd)), device=DEV).to(dt) for _ in range(2)]
    if stride == "padded":
        x = [torch.nn.functional.pad(t, (0, 8, 0, 1))[:, :heads, :hd] for t in x]
    elif stride == "heads first":
        x = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in x]
    n_blocks = rows // block + 3
    shape = hv.Kv4Shape(heads, hd, block, n_blocks)
    pool = torch.full((hv.kv4_pool_bytes(shape),), 0xA5, dtype=torch.uint8, device=DEV)
    assert pool.numel() == n_blocks * heads * ref.chunk_bytes(hd, block)
    slots = rng.permutation(n_blocks * block)[:rows]
    if rows > 4:
        slots[1], slots[3] = -1, n_blocks * block                              # left out
    hv.kv4_append(shape, pool, i32(slots), x[0], x[1], stream=stream())
    want = [c.copy() for c in ref.split_pool(np.full(pool.numel(), 0xA5, np.uint8), heads, hd, block)]
    held = [ref.quantise(f64(t)) for t in x]
    for r, s in enumerate(slots):
        if 0 <= s < n_blocks * block:
            for i, (code, scale) in enumerate(held):
                want[i][s // block, :, s % block] = code[r]
                want[2 + i][s // block, :, s % block] = scale[r]
    got = ref.split_pool(pool.cpu().numpy(), heads, hd, block)
    for g, w, name in zip(got[2:], want[2:], ("key scales", "value scales")):
        np.testing.assert_array_equal(g, w, err_msg=name)
    for i in (0, 1):                                                           # (a zero's sign is not held to anything)
        np.testing.assert_array_equal(np.where(got[i] == 8, 0, got[i]), np.where(want[i] == 8, 0, want[i]))
    # read back, into padded rows; rows left out keep what they had
    out = [torch.full((rows, heads, hd + 8), 7.0, dtype=dt, device=DEV)[:, :, :hd] for _ in range(2)]
    hv.kv4_read(shape, pool, i32(slots), out[0], out[1], stream=stream())
    for o, (code, scale) in zip(out, held):
        back = ref.values(code, scale)
        for r, s in enumerate(slots):
            if not 0 <= s < n_blocks * block:
                back[r] = 7.0
        np.testing.assert_array_equal(f64(o), back)


def test_append_of_no_number():
    """A NaN or an infinity makes its group NaN, and no other."""
    shape = hv.Kv4Shape(2, 128, 16, 1)
    x = torch.randn(3, 2, 128, device=DEV)
    x[0, 0, 5], x[1, 1, 64], x[2, 0, 127] = float("nan"), float("inf"), -float("inf")
    x[2, 1, 0] = 3.4e38
    pool = torch.zeros(hv.kv4_pool_bytes(shape), dtype=torch.uint8, device=DEV)
    hv.kv4_append(shape, pool, i32([0, 1, 2]), x, x, stream=stream())
    k, v = torch.empty_like(x), torch.empty_like(x)
    hv.kv4_read(shape, pool, i32([0, 1, 2]), k, v, stream=stream())
    want = ref.values(*ref.quantise(f64(x)))
    np.testing.assert_array_equal(f64(k), want)
    np.testing.assert_array_equal(f64(v), want)
    assert np.isnan(want).sum() == 3 * 32 and np.isfinite(want[2, 1]).all()


# ---- plan ------------------------------------------------------------------------------------------------------------------------------

class Tables:
    """Tables, list and lengths of n sequences on the GPU."""
    def __init__(self, n, max_blocks, block, n_blocks, max_rows, order=None):
        self.block, self.n_blocks = block, n_blocks
        self.held, self.table, self.status = torch.zeros(n, dtype=torch.int32, device=DEV), torch.full((n, max_blocks), -1, dtype=torch.int32, device=DEV), i32(np.zeros(n))
        self.free = i32([n_blocks] + list(range(n_blocks) if order is None else order))
        self.row_start, self.slots, self.positions = i32(np.zeros(n + 1)), i32(np.zeros(max_rows)), i32(np.zeros(max_rows))

    def plan(self, keep, add):
        hv.kv4_plan(i32(keep) if not torch.is_tensor(keep) else keep, i32(add) if not torch.is_tensor(add) else add, self.held, self.table, self.free, self.row_start, self.slots,
                    self.positions, self.status, block_tokens=self.block, n_blocks=self.n_blocks, stream=stream())

    def now(self):
        return dict(held=self.held.tolist(), table=self.table.tolist(), free=self.free.tolist(), row_start=self.row_start.tolist(), slots=self.slots.tolist(),
                    positions=self.positions.tolist(), status=self.status.tolist())


@pytest.mark.parametrize("n,block,top,scarce", [(1, 16, 5, False), (7, 16, 40, True), (64, 64, 300, False), (100, 32, 90, True), (1025, 16, 20, True), (2300, 128, 400, False)])
def test_plan(n, block, top, scarce):
    rng = random.Random(n)
    max_blocks = -(-4 * top // block)
    n_blocks = max(1, n * max_blocks // (4 if scarce else 1))
    order = list(range(n_blocks))
    rng.shuffle(order)
    max_rows = max(1, n * top // (2 if scarce else 1))
    t = Tables(n, max_blocks, block, n_blocks, max_rows, order)
    length = [0] * n
    for step in range(5):
        before = t.now()
        keep = [rng.choice((x, x, x // 2, 0, max(0, x - 3))) for x in length]
        add = [rng.choice((0, 1, rng.randint(0, top))) for _ in range(n)]
        if step == 3 and n > 4:                                                # requests that cannot be meant
            keep[1], add[2], keep[3], add[4] = -1, -5, 2 ** 31 - 1, 2 ** 31 - 1
        want = ref.plan(keep, add, before["held"], before["table"], before["free"], max_rows, block)
        t.plan(keep, add)
        got = t.now()
        for name in want:
            assert got[name] == want[name], (step, name)
        length = [k + a if s == 0 else x for k, a, s, x in zip(keep, add, want["status"], length)]
        owned = [b for row, h in zip(got["table"], got["held"]) for b in row[:h]] + got["free"][1:1 + got["free"][0]]
        assert sorted(owned) == list(range(n_blocks))                          # every block in one place


def test_plan_with_a_list_that_is_none():
    """A count outside the list gives no block, and nothing is written outside the list."""
    for count in (-3, 2 ** 30):
        t = Tables(2, 4, 16, 8, 64)
        t.free[0] = count
        t.plan([0, 0], [5, 0])
        assert t.status.tolist() == [1, 0] and t.row_start.tolist() == [0, 0, 0] and t.slots.tolist() == [-1] * 64


# ---- attention --------------------------------------------------------------------------------------------------------------------------

class Cache:
    """A pool with sequences of these lengths, their keys and values as held (float64), blocks in random order, NaN wherever nothing is held."""
    def __init__(self, lens, heads, hd, block, seed=0, spare=2):
        rng = np.random.default_rng(seed)
        self.heads, self.hd, self.block, self.lens = heads, hd, block, lens
        nb = [-(-x // block) for x in lens]
        self.n_blocks, self.max_blocks = sum(nb) + spare, max(nb + [1])
        perm = rng.permutation(self.n_blocks)
        self.table = np.full((len(lens), self.max_blocks), -1, np.int32)
        parts = [np.full((self.n_blocks, heads, block, w), f, np.uint8) for w, f in ((hd, 15), (hd, 15), (hd // 32, 255), (hd // 32, 255))]
        self.k, self.v, at = [], [], 0
        for s, x in enumerate(lens):
            self.table[s, :nb[s]] = perm[at:at + nb[s]]
            at += nb[s]
            pos = np.arange(x)
            b, r = self.table[s, pos // block], pos % block
            for i in (0, 1):
                code, scale = ref.quantise(rng.standard_normal((x, heads, hd)) * np.exp(0.5 * rng.standard_normal((1, heads, hd))))
                parts[i][b, :, r], parts[2 + i][b, :, r] = code, scale
        self.parts = parts
        self.upload()

    def upload(self):
        self.pool = torch.as_tensor(ref.join_pool(*self.parts), device=DEV)
        self.k, self.v = [], []
        for s, x in enumerate(self.lens):
            pos = np.arange(x)
            b, r = self.table[s, pos // self.block], pos % self.block
            self.k.append(ref.values(self.parts[0][b, :, r], self.parts[2][b, :, r]))
            self.v.append(ref.values(self.parts[1][b, :, r], self.parts[3][b, :, r]))

    @property
    def shape(self):
        return hv.Kv4Shape(self.heads, self.hd, self.block, self.n_blocks)


def causal(rows, length):
    return np.arange(length)[None] <= np.arange(rows)[:, None] + length - rows


def masked(bits, length):
    new = np.arange(length)[None] - (length - len(bits))
    return (new < 0) | ((np.asarray(bits, dtype=np.uint64)[:, None] >> np.maximum(new, 0).astype(np.uint64)) & np.uint64(1)).astype(bool)


def attend(cache, rows, q, out=None, mask=None, scale=None, max_len=None, row_start=None, workspace=None, table=None, max_rows=None):
    out = torch.full_like(q, 9.0) if out is None else out
    starts = np.concatenate([[0], np.cumsum(rows)]) if row_start is None else row_start
    top = max(list(rows) + [1]) if max_rows is None else max_rows
    length = max(cache.lens + [1]) if max_len is None else max_len
    if workspace is None:
        workspace = torch.zeros(hv.kv4_attend_bytes(cache.shape, q.shape[1], len(rows), top, length, q.dtype), dtype=torch.uint8, device=DEV)
    hv.kv4_attend(cache.shape, cache.pool, i32(cache.table if table is None else table), i32(starts), i32(cache.lens), q, out, max_rows=top, max_len=length, workspace=workspace, scale=scale,
                  mask=None if mask is None else torch.as_tensor(np.asarray(mask, np.uint64).view(np.int64), device=DEV), stream=stream())
    return out


def check(cache, rows, q, out, kind, see=None, scale=None):
    scale = cache.hd ** -0.5 if scale is None else scale
    got, at = f64(out), 0
    for s, r in enumerate(rows):
        on = see[s] if see is not None else causal(r, cache.lens[s])
        want, tol = ref.attend(f64(q)[at:at + r], cache.k[s], cache.v[s], on, scale, kind)
        miss = np.abs(got[at:at + r] - want) / np.maximum(tol, 1e-30)
        bad = ~np.isfinite(got[at:at + r])
        assert not bad.any(), (s, "not finite", np.argwhere(bad)[:4])
        empty = ~on.any(-1)
        assert (got[at:at + r][empty] == 0).all()
        assert miss[~empty].max(initial=0) <= 1, (s, float(miss[~empty].max()))
        at += r


SHAPES = [                                                                     # heads, group, hd, block, lens, rows
    (1, 1, 64, 16, [1], [1]),
    (2, 1, 128, 16, [15, 16, 17, 31, 32, 33], [1, 1, 1, 1, 1, 1]),
    (4, 1, 64, 32, [65, 0, 1, 127, 129, 300], [1, 0, 1, 5, 8, 16]),
    (4, 7, 128, 64, [100, 1120, 64], [7, 7, 1]),
    (2, 8, 128, 128, [700, 3, 129], [1, 3, 1]),
    (8, 2, 64, 256, [513, 256, 255, 40], [9, 17, 1, 40]),
    (1, 3, 128, 32, [61, 200], [61, 33]),
    (3, 1, 128, 64, [650], [6]),
    (2, 16, 64, 16, [2000, 5], [2, 2]),
    (2, 1, 128, 64, [290, 131], [290, 65]),
    (2, 4, 128, 32, [500, 77], [400, 77]),
    (1, 2, 64, 64, [700], [700]),
]


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("heads,group,hd,block,lens,rows", SHAPES)
def test_attend(kind, heads, group, hd, block, lens, rows):
    cache = Cache(lens, heads, hd, block, seed=sum(lens))
    g = torch.Generator(device=DEV).manual_seed(len(lens))
    q = torch.randn(sum(rows), heads * group, hd, generator=g, device=DEV).to(getattr(torch, kind))
    check(cache, rows, q, attend(cache, rows, q), kind)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("pairs,length", [(16, 1 << 20), (2000, 64), (1000000, 1), (1000000, 300)])
@pytest.mark.parametrize("heads,group,hd,block,lens,rows", SHAPES)
def test_attend_forms(kind, heads, group, hd, block, lens, rows, pairs, length):
    """The same calls as launched for other sizes: which kernel runs is a matter of the promised rows and lengths, the results are not."""
    cache = Cache(lens, heads, hd, block, seed=sum(lens))
    g = torch.Generator(device=DEV).manual_seed(len(lens))
    q = torch.randn(sum(rows), heads * group, hd, generator=g, device=DEV).to(getattr(torch, kind))
    check(cache, rows, q, attend(cache, rows, q, max_rows=max(max(rows), pairs // group), max_len=length), kind)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("heads,group,hd", [(2, 1, 64), (1, 3, 128)])
def test_attend_many_sequences(kind, heads, group, hd):
    """More sequences than lanes, empty ones among them; trees of 64 rows in enough sequences for the prompts' kernels."""
    rng = random.Random(hd)
    lens = [rng.choice((0, 1, 16, 40, rng.randrange(200))) for _ in range(150)]
    rows = [min(n, rng.choice((0, 1, 1, 3))) for n in lens]
    cache = Cache(lens, heads, hd, 16, seed=8)
    q = torch.randn(sum(rows), heads * group, hd, device=DEV).to(getattr(torch, kind))
    check(cache, rows, q, attend(cache, rows, q), kind)
    cache = Cache([64 + s % 9 for s in range(96)], 8, 64, 32, seed=9)
    bits = [tree_bits(64, s) for s in range(96)]
    q = torch.randn(96 * 64, 16, 64, device=DEV).to(getattr(torch, kind))
    check(cache, [64] * 96, q, attend(cache, [64] * 96, q, mask=sum(bits, [])), kind, see=[masked(b, n) for b, n in zip(bits, cache.lens)])


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_attend_scores_of_any_size(kind):
    """Scores far below zero alone, and a scale of zero and below it."""
    cache = Cache([40], 1, 64, 16, seed=12)
    q = torch.randn(3, 1, 64, device=DEV).to(getattr(torch, kind))
    for scale in (0.0, -0.125):
        for pairs in (3, 1000000):
            check(cache, [3], q, attend(cache, [3], q, scale=scale, max_rows=pairs), kind, scale=scale)
    cache.parts[0][:] = (cache.parts[0] & 0x77) | 0x11                         # keys above zero: the scores of queries below it are far below it, all of them
    cache.upload()
    q = -q.abs() * 2.0 ** 70
    for pairs in (3, 2000, 1000000):
        out = attend(cache, [3], q, scale=2.0 ** 40, max_rows=pairs)
        assert torch.isfinite(out).all() and (out != 0).any()
        check(cache, [3], q, out, kind, scale=2.0 ** 40)


def test_workspace_is_left_as_found():
    """One workspace for calls of any sizes, of attention and of log probabilities, in any order: as with one of their own."""
    calls = []
    for lens, rows, heads, group in (([700], [1], 4, 1), ([3000, 90], [3, 8], 8, 2), ([130] * 5, [1] * 5, 2, 4), ([50], [50], 1, 1)):
        cache = Cache(lens, heads, 128, 32, seed=len(lens))
        q = torch.randn(sum(rows), heads * group, 128, device=DEV)
        calls.append(lambda ws, c=cache, r=rows, q=q: [attend(c, r, q, workspace=ws)])
    for rows, vocab in ((1, 90000), (40, 20000), (3, 30000)):
        x, tokens = torch.randn(rows, vocab, device=DEV), i32(np.arange(rows)[:, None])

        def call(ws, x=x, tokens=tokens, rows=rows, vocab=vocab):
            lp, ids, tlp = torch.empty(rows, 1, device=DEV), torch.empty(rows, 4, dtype=torch.int32, device=DEV), torch.empty(rows, 4, device=DEV)
            hv.logprobs(x, tokens, lp, None, ids, tlp, workspace=torch.zeros(hv.logprobs_bytes(rows, vocab, 4), dtype=torch.uint8, device=DEV) if ws is None else ws, stream=stream())
            return [lp, ids, tlp]
        calls.append(call)
    want = [c(None) for c in calls]
    ws = torch.zeros(1 << 25, dtype=torch.uint8, device=DEV)
    order = [i for i in range(len(calls))] * 6
    random.Random(3).shuffle(order)
    for i in order:
        for a, b in zip(want[i], calls[i](ws)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_attend_large_scores_and_scale(kind):
    """Scores far apart (one weight takes all) and a scale of the caller's; fewer cached rows promised than there are."""
    cache = Cache([400, 35], 2, 128, 32, seed=5)
    q = (30 * torch.randn(3, 4, 128, device=DEV)).to(getattr(torch, kind))
    check(cache, [2, 1], q, attend(cache, [2, 1], q), kind)
    check(cache, [2, 1], q, attend(cache, [2, 1], q, scale=0.003, max_len=17), kind, scale=0.003)


def tree_bits(n, seed):
    rng, bits = random.Random(seed), []
    for i in range(n):
        bits.append((bits[rng.randrange(i)] if i else 0) | 1 << i)
    return bits


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("heads,group,hd,lens,rows", [(2, 1, 128, [300], [64]), (4, 7, 128, [161, 61], [61, 61]), (2, 2, 64, [64, 90, 20], [3, 40, 20])])
def test_attend_tree(kind, heads, group, hd, lens, rows):
    cache = Cache(lens, heads, hd, 16, seed=1)
    bits = [tree_bits(r, s) for s, r in enumerate(rows)]
    q = torch.randn(sum(rows), heads * group, hd, device=DEV).to(getattr(torch, kind))
    out = attend(cache, rows, q, mask=sum(bits, []))
    check(cache, rows, q, out, kind, see=[masked(b, n) for b, n in zip(bits, lens)])


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_attend_rows_that_see_nothing(kind):
    """Empty caches, masks without a bit, more rows than cached ones: zeros; rows of no sequence stay as they were."""
    cache = Cache([0, 5, 3, 40], 2, 64, 16, seed=2)
    rows = [2, 5, 6, 3]
    q = torch.randn(20, 2, 64, device=DEV).to(getattr(torch, kind))
    bits = [0, 0] + [0, 1, 0, 8, 31] + [0] * 6 + [0, 0, 1]
    see = [masked(b, n) for b, n in zip((bits[:2], bits[2:7], bits[7:13], bits[13:]), cache.lens)]
    out = attend(cache, rows, q, mask=bits + [~0 & 2 ** 64 - 1] * 4)
    check(cache, rows, q[:16], out[:16], kind, see=see)
    assert (out[16:] == 9).all()
    assert (out[:2] == 0).all() and (out[2] == 0).all() and (out[13] != 0).any()
    out = attend(cache, rows, q)                                               # causal: the first three of six rows stand before the cache
    check(cache, rows, q[:16], out[:16], kind)
    assert (out[7:10] == 0).all() and (out[10:13] != 0).any() and (out[16:] == 9).all()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("group,rows", [(1, 6), (2, 40)])
def test_attend_nan_reaches_only_rows_that_see_it(kind, group, rows):
    cache = Cache([70], 2, 128, 16, seed=3)
    b, r = cache.table[0, 68 // 16], 68 % 16                                   # the last row but one: seen by the last two rows alone
    for part in (2, 3):
        keep = [p.copy() for p in cache.parts]
        cache.parts[part][b, 0, r, 1] = 255
        cache.pool = torch.as_tensor(ref.join_pool(*cache.parts), device=DEV)
        q = torch.randn(rows, 2 * group, 128, device=DEV).to(getattr(torch, kind))
        out = attend(cache, [rows], q)
        cache.parts = keep
        cache.upload()
        check(cache, [rows - 2], q[:rows - 2], out[:rows - 2], kind, see=[causal(rows, 70)[:rows - 2]])
        nan = torch.isnan(out[rows - 2:])
        assert not nan[:, group:].any()                                        # the other key head
        if part == 2:
            assert nan[:, :group].all()                                        # a score: the whole row
        else:
            assert nan[:, :group, 32:64].all() and not nan[:, :group, :32].any() and not nan[:, :group, 64:].any()


def test_attend_blocks_outside_the_pool():
    """Table entries that are no block: their keys are left out."""
    cache = Cache([100], 1, 64, 16, seed=4)
    q = torch.randn(2, 1, 64, device=DEV)
    table = cache.table.copy()
    table[0, 2], table[0, 4] = -7, cache.n_blocks
    out = attend(cache, [2], q, table=table)
    on = causal(2, 100) & ~np.isin(np.arange(100) // 16, (2, 4))[None]
    check(cache, [2], q, out, "float32", see=[on])


@pytest.mark.parametrize("pairs", [2, 2000, 1000000])
def test_attend_lengths_that_are_none(pairs):
    """Cached rows below zero, and more than the table holds: as zero, and as many as it holds."""
    cache = Cache([64, 0, 0], 1, 64, 16, seed=4)
    q = torch.randn(6, 1, 64, device=DEV)
    cache.lens = [2 ** 31 - 1, -2 ** 31, -1]
    out = attend(cache, [2, 2, 2], q, max_len=64, max_rows=pairs)
    assert not out[2:].any()
    cache.lens = [64, 0, 0]
    check(cache, [2, 2, 2], q, out, "float32")


def test_attend_rows_outside_the_call():
    """A row_start that does not fit the rows of q: the sequence is left out."""
    cache = Cache([40, 40], 1, 64, 16, seed=4)
    q = torch.randn(4, 1, 64, device=DEV)
    out = attend(cache, [2, 2], q, row_start=[0, 2, 5])
    check(cache, [2], q[:2], out[:2], "float32")
    assert (out[2:] == 9).all()
    out = attend(cache, [2, 2], q, row_start=[-1, 2, 4])
    assert (out[:2] == 9).all() and (out[2:] != 9).all()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_attend_strides(kind):
    """Rows of q inside wider rows (q|k|v side by side), rows of out inside wider ones."""
    cache = Cache([90, 30], 2, 64, 32, seed=6)
    wide = torch.randn(4, 12, 64, device=DEV).to(getattr(torch, kind))
    q = wide[:, 2:8]
    out = torch.full((4, 9, 64), 9.0, device=DEV).to(getattr(torch, kind))
    attend(cache, [1, 3], q, out=out[:, 1:7])
    check(cache, [1, 3], q, out[:, 1:7], kind)
    assert (out[:, 0] == 9).all() and (out[:, 7:] == 9).all()


@pytest.mark.parametrize("rows", [1, 200])
def test_attend_in_a_pool_beyond_4_gib(rows):
    """Blocks whose bytes lie beyond 2^32."""
    heads, hd, block = 8, 128, 64
    chunk = heads * ref.chunk_bytes(hd, block)
    n_blocks = (2 ** 32 + 2 ** 28) // chunk
    small = Cache([500], heads, hd, block, seed=7, spare=0)
    pool = torch.empty(n_blocks * chunk, dtype=torch.uint8, device=DEV)
    table = i32(n_blocks - 1 - small.table)
    for b in range(small.n_blocks):
        pool[(n_blocks - 1 - b) * chunk:(n_blocks - b) * chunk] = small.pool[b * chunk:(b + 1) * chunk]
    q = torch.randn(rows, heads, hd, device=DEV)
    out = torch.empty_like(q)
    shape = hv.Kv4Shape(heads, hd, block, n_blocks)
    ws = torch.zeros(hv.kv4_attend_bytes(shape, heads, 1, rows, 500, q.dtype), dtype=torch.uint8, device=DEV)
    hv.kv4_attend(shape, pool, table, i32([0, rows]), i32([500]), q, out, max_rows=rows, max_len=500, workspace=ws, stream=stream())
    check(small, [rows], q, out, "float32")
    # a row written to the last slot and read back
    x = torch.randn(1, heads, hd, device=DEV)
    k, v = torch.empty_like(x), torch.empty_like(x)
    last = i32([n_blocks * block - 1])
    hv.kv4_append(shape, pool, last, x, x, stream=stream())
    hv.kv4_read(shape, pool, last, k, v, stream=stream())
    np.testing.assert_array_equal(f64(k), ref.values(*ref.quantise(f64(x))))


# ---- log probabilities ----------------------------------------------------------------------------------------------------------------

def run_logprobs(x, tokens, temperature=1.0, top=0, entropy=True):
    rows, V = x.shape
    ws = torch.zeros(hv.logprobs_bytes(rows, V, top), dtype=torch.uint8, device=DEV)
    lp = torch.full((rows, tokens.shape[1]), 9.0, device=DEV)
    h = torch.full((rows,), 9.0, device=DEV) if entropy else None
    ids = torch.full((rows, top), 9, dtype=torch.int32, device=DEV) if top else None
    tlp = torch.full((rows, top), 9.0, device=DEV) if top else None
    hv.logprobs(x, i32(tokens), lp, h, ids, tlp, temperature=temperature, workspace=ws, stream=stream())
    return lp, h, ids, tlp


def check_logprobs(x, tokens, temperature, top, got):
    """Relative to half a step u of fp32: (x - max) and its scaling by 1 / T are off by 3 u |y|, the exponential by 4 u, a sum of V of them by (V / 16 + 64) u at
    most in its order (16 or more partial sums); the logarithm and the last subtraction by 2 u of their sizes."""
    lp, h, ids, tlp = got
    want = ref.logprobs(f64(x), np.asarray(tokens), temperature, top)
    u = ref.U["float32"]
    y = f64(x) / temperature
    y = np.where(np.isfinite(y), y, 0)
    span = (y.max(-1) - y.min(-1))[:, None] + 1
    tol = u * (8 * span + x.shape[1] / 16 + 64)
    for a, b in ((lp, want[0]), (tlp, want[3])):
        if a is None:
            continue
        g = f64(a)
        assert (np.isnan(g) == np.isnan(b)).all()
        inf = np.isinf(b)
        assert (g[inf] == b[inf]).all()
        ok = ~np.isnan(b) & ~inf
        assert (np.abs(g - np.where(ok, b, 0)) <= tol + 4 * u * np.abs(np.where(ok, b, 0)))[ok].all()
    if h is not None:
        g, ok = f64(h), ~np.isnan(want[1])
        assert (np.isnan(g) == ~ok).all()
        assert (np.abs(g - np.where(ok, want[1], 0)) <= 2 * tol[:, 0] * (1 + np.log(x.shape[1])))[ok].all()
    if ids is not None:
        np.testing.assert_array_equal(ids.cpu().numpy(), want[2])


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,vocab,n,top,temperature", [(1, 1, 1, 1, 1.0), (3, 5, 2, 5, 0.5), (2, 1024, 1, 20, 1.0), (6, 32000, 1, 5, 1.0), (1, 152064, 3, 32, 0.7), (130, 4097, 1, 0, 2.0), (17, 50257, 4, 7, 1.3), (300, 999, 2, 32, 1.0), (2, 3001, 300, 3, 1.0)])
def test_logprobs(kind, rows, vocab, n, top, temperature):
    g = torch.Generator(device=DEV).manual_seed(vocab)
    x = (3 * torch.randn(rows, vocab, generator=g, device=DEV)).to(getattr(torch, kind))
    tokens = torch.randint(0, vocab, (rows, n), generator=g, device=DEV).cpu().numpy()
    check_logprobs(x, tokens, temperature, top, run_logprobs(x, tokens, temperature, top))


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [40, 5000, 70000])
def test_logprobs_ties_and_order(kind, vocab):
    """All logits equal, few distinct ones, rising and falling rows, -0 beside 0: the lower id first."""
    dt = getattr(torch, kind)
    i = torch.arange(vocab, device=DEV)
    x = torch.stack([torch.zeros(vocab, device=DEV), (i % 3).float(), i.float() / vocab, -i.float() / vocab, torch.where(i % 2 == 0, -0.0, 0.0), torch.where(i == vocab - 1, 50.0, -50.0)]).to(dt)
    tokens = np.array([[0, vocab - 1]] * len(x))
    check_logprobs(x, tokens, 1.0, 32, run_logprobs(x, tokens, 1.0, 32))


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_logprobs_masked_and_broken_rows(kind):
    """-inf and the type's lowest value on all but a few tokens; rows without a finite maximum or with a NaN; tokens outside the vocabulary."""
    dt = getattr(torch, kind)
    x = torch.randn(7, 9001, device=DEV).to(dt)
    x[0, 3:] = -math.inf
    x[1, 5:] = torch.finfo(dt).min
    x[2] = -math.inf
    x[3, 77] = math.nan
    x[4, 8000] = math.inf
    x[5, :9000] = -math.inf
    tokens = np.array([[0, 8000, -1], [1, 6, 9001], [0, 1, 2], [0, 77, 5], [8000, 1, 2], [9000, 0, 2 ** 31 - 1], [5, -2 ** 31, 7]])
    got = run_logprobs(x, tokens, 1.0, 4)
    lp, h, ids, tlp = (f64(t) for t in got)
    want = ref.logprobs(f64(x), tokens, 1.0, 4)
    np.testing.assert_array_equal(ids, want[2])
    tol = 2.0 ** -24 * (9001 / 16 + 200)
    for g, w in ((lp, want[0]), (tlp, want[3]), (h, want[1])):
        np.testing.assert_array_equal(np.isnan(g), np.isnan(w))
        np.testing.assert_array_equal(g[np.isinf(w)], w[np.isinf(w)])
        ok = np.isfinite(w)
        assert (np.abs(g - np.where(ok, w, 0)) <= tol * (2 + np.abs(np.where(ok, w, 0))))[ok].all()


def test_logprobs_of_rows_inside_wider_ones():
    wide = torch.randn(5, 4000, device=DEV)
    x = wide[:, 3:1004]
    tokens = np.arange(5)[:, None] * 200
    check_logprobs(x, tokens, 1.0, 6, run_logprobs(x, tokens, 1.0, 6))
    check_logprobs(x.to(torch.bfloat16)[:, 1:], tokens, 1.0, 6, run_logprobs(x.to(torch.bfloat16)[:, 1:], tokens, 1.0, 6))
    run_logprobs(x, tokens, 1.0, 0, entropy=False)


# ---- together, streams, graphs ----------------------------------------------------------------------------------------------------------

def serve(steps, heads=2, group=2, hd=64, block=16, use=stream):
    """Three conversations through plan, append, attend and log probabilities; some rows of every step are given back."""
    g = torch.Generator(device=DEV).manual_seed(11)
    n, max_blocks, n_blocks = 3, 12, 30
    t = Tables(n, max_blocks, block, n_blocks, 120)
    shape = hv.Kv4Shape(heads, hd, block, n_blocks)
    pool = torch.full((hv.kv4_pool_bytes(shape),), 255, dtype=torch.uint8, device=DEV)
    head = torch.randn(heads * group * hd, 500, generator=g, device=DEV)
    ws = torch.zeros(hv.kv4_attend_bytes(shape, heads * group, n, 40, max_blocks * block, torch.float32), dtype=torch.uint8, device=DEV)
    ws2 = torch.zeros(hv.logprobs_bytes(120, 500, 3), dtype=torch.uint8, device=DEV)
    held = [[], [], []]                                                        # what a dense program would keep: (k, v) rows as held
    results = []
    for step in range(steps):
        add = [40, 17, 1] if step == 0 else [5, 5, 5]
        keep = [len(x) for x in held]
        t.plan(keep, add)
        rows = sum(add)
        k, v, q = (torch.randn(120, w, hd, generator=g, device=DEV) for w in (heads, heads, heads * group))
        hv.kv4_append(shape, pool, t.slots, k, v, stream=use())                # (rows behind the last: slot -1)
        out = torch.zeros(120, heads * group, hd, device=DEV)
        lens = i32([a + b for a, b in zip(keep, add)])
        hv.kv4_attend(shape, pool, t.table, t.row_start, lens, q, out, max_rows=40, max_len=max_blocks * block, workspace=ws, stream=use())
        logits = out.reshape(120, -1) @ head
        lp, h, ids, tlp = torch.empty(120, 1, device=DEV), torch.empty(120, device=DEV), torch.empty(120, 3, dtype=torch.int32, device=DEV), torch.empty(120, 3, device=DEV)
        hv.logprobs(logits, torch.zeros(120, 1, dtype=torch.int32, device=DEV), lp, h, ids, tlp, workspace=ws2, stream=use())
        assert t.status.tolist() == [0, 0, 0]
        at = 0
        for s in range(n):
            ks, vs = (ref.values(*ref.quantise(f64(x[at:at + add[s]]))) for x in (k, v))
            held[s] += list(zip(ks, vs))
            dense_k, dense_v = np.stack([x[0] for x in held[s]]), np.stack([x[1] for x in held[s]])
            want, tol = ref.attend(f64(q[at:at + add[s]]), dense_k, dense_v, causal(add[s], len(held[s])), hd ** -0.5, "float32")
            assert (np.abs(f64(out[at:at + add[s]]) - want) <= tol).all(), (step, s)
            at += add[s]
            del held[s][len(held[s]) - (0 if step == 0 else (step + s) % 5):]  # rejected drafts
        assert not out[rows:].any()
        check_logprobs(logits, np.zeros((120, 1), int), 1.0, 3, (lp, h, ids, tlp))
        results.append((out.clone(), lp.clone()))
    return results


def test_together():
    serve(6)


def test_together_on_another_stream():
    want = serve(3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = serve(3)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("rows,heads,group", [(1, 4, 1), (8, 2, 7), (130, 1, 2)])
def test_graph_replays(rows, heads, group):
    """plan, append, attend and logprobs captured once; lengths, rows and queries change between replays, with eager calls in between."""
    hd, block, top = 64, 16, 400
    n = 2
    t = Tables(n, -(-top // block), block, 60, n * rows)
    shape = hv.Kv4Shape(heads, hd, block, 60)
    pool = torch.full((hv.kv4_pool_bytes(shape),), 255, dtype=torch.uint8, device=DEV)
    keep, add, lens = i32([0, 0]), i32([rows, rows]), i32([rows, rows])
    k, v, q = (torch.zeros(n * rows, w, hd, device=DEV) for w in (heads, heads, heads * group))
    out = torch.zeros_like(q)
    space = lambda: torch.zeros(hv.kv4_attend_bytes(shape, heads * group, n, rows, top, torch.float32), dtype=torch.uint8, device=DEV)
    ws, ws_eager = space(), space()
    lp, ids, tlp = torch.empty(n * rows, 1, device=DEV), torch.empty(n * rows, 2, dtype=torch.int32, device=DEV), torch.empty(n * rows, 2, device=DEV)
    ws2 = torch.zeros(hv.logprobs_bytes(n * rows, heads * group * hd, 2), dtype=torch.uint8, device=DEV)
    tokens = torch.zeros(n * rows, 1, dtype=torch.int32, device=DEV)

    def call():
        t.plan(keep, add)
        hv.kv4_append(shape, pool, t.slots, k, v, stream=stream())
        hv.kv4_attend(shape, pool, t.table, t.row_start, lens, q, out, max_rows=rows, max_len=top, workspace=ws, stream=stream())
        hv.logprobs(out.view(n * rows, -1), tokens, lp, None, ids, tlp, workspace=ws2, stream=stream())

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    dense = [[], []]
    for step in range(3):
        for x in (k, v, q):
            x.normal_()
        start = [len(d) for d in dense]
        keep.copy_(i32(start))
        lens.copy_(i32([s + rows for s in start]))
        graph.replay()
        torch.cuda.synchronize()
        assert t.status.tolist() == [0, 0]
        again = torch.empty_like(out)
        hv.kv4_attend(shape, pool, t.table, t.row_start, lens, q, again, max_rows=rows, max_len=top, workspace=ws_eager, stream=stream())
        assert torch.equal(again, out)
        check_logprobs(out.view(n * rows, -1), np.zeros((n * rows, 1), int), 1.0, 2, (lp, None, ids, tlp))
        for s in range(n):
            part = slice(s * rows, (s + 1) * rows)
            dense[s] += list(zip(*(ref.values(*ref.quantise(f64(x[part]))) for x in (k, v))))
            want, tol = ref.attend(f64(q[part]), np.stack([x[0] for x in dense[s]]), np.stack([x[1] for x in dense[s]]), causal(rows, len(dense[s])), hd ** -0.5, "float32")
            assert (np.abs(f64(out[part]) - want) <= tol).all(), (step, s)
            del dense[s][max(1, len(dense[s]) - rows // 2):]


def test_host_memory_is_refused():
    """Addresses that are no device memory of the current device."""
    shape = hv.Kv4Shape(1, 64, 16, 4)
    pool = torch.zeros(hv.kv4_pool_bytes(shape), dtype=torch.uint8, device=DEV)
    x = torch.zeros(2, 1, 64, device=DEV)
    for args in ((pool.cpu(), i32([0, 1]), x, x), (pool, i32([0, 1]).cpu(), x, x), (pool, i32([0, 1]), x.cpu(), x.cpu()), (pool, i32([0, 1]), x.cpu().pin_memory(), x)):
        with pytest.raises(hv.HivisError) as e:
            hv.kv4_append(shape, *args, stream=stream())
        assert e.value.code == hv.HIVIS_EINVAL and "device memory" in str(e.value)
    with pytest.raises(hv.HivisError):
        hv.logprobs(torch.zeros(1, 64), i32([[0]]), torch.zeros(1, 1, device=DEV), workspace=torch.zeros(1 << 16, dtype=torch.uint8, device=DEV), stream=stream())


def test_workspace_too_small_is_refused():
    cache = Cache([3000], 2, 64, 16, seed=1)
    q = torch.zeros(4, 2, 64, device=DEV)
    with pytest.raises(hv.HivisError) as e:
        attend(cache, [4], q, workspace=torch.zeros(15, dtype=torch.uint8, device=DEV))
    assert e.value.code == hv.HIVIS_EINVAL and "workspace" in str(e.value)
