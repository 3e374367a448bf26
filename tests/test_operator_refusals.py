"""What the operators on callers' tensors refuse before they look at a device (no GPU needed), through the C entry points and the binding."""
import ctypes as C

import numpy as np
import pytest

from paper_2509_23928_amd import HIVIS_BF16, HIVIS_EINVAL, HIVIS_F32, HivisError, Kv4Shape, binding

LIB = binding.load_library()
P = C.c_void_p(0x1000)                     # an address that nothing looks at: the arguments beside it are refused first


def refused(rc, *words):
    text = LIB.hivis_last_error(None).decode()
    assert rc == HIVIS_EINVAL and all(w in text for w in words), (rc, text)


@pytest.mark.parametrize("shape,word", [((0, 64, 16, 1), "n_kv_heads"), ((1, 96, 16, 1), "head_dim"), ((1, 64, 8, 1), "block_tokens"), ((1, 64, 48, 1), "block_tokens"),
                                        ((1, 64, 512, 1), "block_tokens"), ((1, 64, 16, 0), "n_blocks"), ((1, 64, 256, 1 << 24), "n_blocks"), ((-1, 64, 16, 1), "n_kv_heads")])
def test_shapes(shape, word):
    s = Kv4Shape(*shape)
    refused(LIB.hivis_kv4_pool_bytes(C.byref(s)), word)
    refused(LIB.hivis_kv4_append(None, C.byref(s), HIVIS_F32, P, P, 64, 64, 1, P, P), word)
    refused(LIB.hivis_kv4_read(None, C.byref(s), HIVIS_F32, P, 1, P, P, P, 64, 64), word)
    refused(LIB.hivis_kv4_attend_bytes(C.byref(binding.hivis_kv4_attention(cache=s, n_q_heads=1, n_seqs=1))), word)
    refused(LIB.hivis_kv4_attend(None, C.byref(binding.hivis_kv4_attention(cache=s, n_q_heads=1, n_seqs=1))), word)
    refused(LIB.hivis_kv4_pool_bytes(None), "null")


def test_pool_bytes():
    assert LIB.hivis_kv4_pool_bytes(C.byref(Kv4Shape(8, 128, 64, 1000))) == 1000 * 8 * 64 * 136
    assert LIB.hivis_kv4_pool_bytes(C.byref(Kv4Shape(40, 64, 256, 8388607))) == 8388607 * 40 * 256 * 68


def test_plan():
    def call(n=1, blocks=4, T=16, pool=8, rows=5, keep=P, table=P, slots=P, status=P):
        return LIB.hivis_kv4_plan(None, n, blocks, T, pool, keep, P, P, table, P, P, slots, None, rows, status)
    refused(call(n=0), "n_seqs")
    refused(call(n=-4), "n_seqs")
    refused(call(blocks=0), "max_blocks")
    refused(call(blocks=1 << 27), "max_blocks")
    refused(call(T=20), "block_tokens")
    refused(call(pool=0), "n_blocks")
    refused(call(rows=-1), "max_rows")
    refused(call(n=1 << 20, blocks=1 << 12), "n_seqs")
    for name in ("keep", "table", "slots", "status"):
        refused(call(**{name: None}), "null")


@pytest.mark.parametrize("call", ["append", "read"])
def test_rows(call):
    s = Kv4Shape(2, 64, 16, 4)

    def run(dtype=HIVIS_F32, k=P, v=P, row=128, head=64, n=1, slots=P, pool=P):
        if call == "append":
            return LIB.hivis_kv4_append(None, C.byref(s), dtype, k, v, row, head, n, slots, pool)
        return LIB.hivis_kv4_read(None, C.byref(s), dtype, pool, n, slots, k, v, row, head)
    refused(run(dtype=2), "dtype")
    refused(run(n=-1), "n_rows")
    refused(run(n=(1 << 30) + 1), "n_rows")
    refused(run(row=132), "strides")
    refused(run(head=66), "strides")
    refused(run(head=56), "strides")
    refused(run(row=-128), "strides")
    refused(run(k=C.c_void_p(0x1004)), "16 bytes")
    refused(run(pool=C.c_void_p(0x1008)), "pool")
    for name in ("k", "v", "slots", "pool"):
        refused(run(**{name: None}), "null")


def test_attend():
    good = dict(cache=Kv4Shape(2, 64, 16, 4), dtype=HIVIS_BF16, n_q_heads=4, n_seqs=1, n_rows=1, max_blocks=2, max_rows=1, max_len=20, scale=1.0, pool=P, table=P, row_start=P, kv_len=P, q=P, q_stride=256,
                mask=None, out=P, out_stride=256, workspace=P, workspace_bytes=1 << 30)

    def call(**kw):
        a = binding.hivis_kv4_attention(**{k: v for k, v in dict(good, **kw).items() if v is not None})
        return LIB.hivis_kv4_attend(None, C.byref(a))
    refused(LIB.hivis_kv4_attend(None, None), "null")
    refused(call(dtype=7), "dtype")
    refused(call(n_q_heads=3), "n_q_heads")
    refused(call(n_q_heads=0), "n_q_heads")
    refused(call(n_seqs=-1), "n_seqs")
    refused(call(n_rows=-1), "n_rows")
    refused(call(max_blocks=0), "max_blocks")
    refused(call(max_blocks=1 << 28), "max_blocks")
    refused(call(max_rows=-1), "max_rows")
    refused(call(max_rows=65, mask=P), "mask")
    refused(call(scale=float("nan")), "scale")
    refused(call(scale=float("inf")), "scale")
    refused(call(q_stride=252), "strides")
    refused(call(out_stride=248), "strides")
    refused(call(out_stride=260), "strides")
    refused(call(q=C.c_void_p(0x1008)), "16 bytes")
    refused(call(workspace_bytes=0), "workspace")
    for name in ("pool", "table", "row_start", "kv_len", "q", "out", "workspace"):
        refused(call(**{name: None}), "null")
    assert call(n_seqs=0) == 0 and call(max_rows=0) == 0 and call(n_rows=0) == 0       # nothing to do


def test_logprobs():
    def call(dtype=HIVIS_F32, x=P, ld=100, rows=1, vocab=100, T=1.0, tokens=P, n=1, lp=P, top=2, ids=P, tlp=P, ws=P, room=1 << 30):
        return LIB.hivis_logprobs(None, dtype, x, ld, rows, vocab, T, tokens, n, lp, None, top, ids, tlp, ws, room)
    refused(call(dtype=5), "dtype")
    refused(call(ld=99), "row_stride")
    refused(call(rows=-1), "n_rows")
    refused(call(vocab=0, ld=0), "vocab")
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-42):
        refused(call(T=T), "temperature")
    refused(call(top=33), "top_k")
    refused(call(top=-1), "top_k")
    refused(call(vocab=1, top=2), "top_k")
    refused(call(n=-1), "null")
    refused(call(room=0), "workspace")
    refused(call(x=C.c_void_p(0x1002)), "start")
    for name in ("x", "tokens", "lp", "ids", "tlp", "ws"):
        refused(call(**{name: None}), "null")
    refused(LIB.hivis_logprobs_bytes(-1, 5, 0), "n_rows")
    assert call(rows=0) == 0


def test_the_binding_checks_types_and_shapes():
    torch = pytest.importorskip("torch")
    s = Kv4Shape(2, 64, 16, 4)
    pool, slots, x = torch.zeros(binding.kv4_pool_bytes(s), dtype=torch.uint8), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 2, 64)
    bad = [(pool[:-1], slots, x, x), (pool.to(torch.int8), slots, x, x), (pool, slots.long(), x, x), (pool, slots, x[:2], x[:2]), (pool, slots, x, x.bfloat16()), (pool, slots, x.half(), x.half()),
           (pool, slots, x.transpose(1, 2).contiguous().transpose(1, 2), x), (pool, slots, torch.zeros(3, 2, 128)[:, :, :64], x)]
    for args in bad:
        for call in (binding.kv4_append, binding.kv4_read):
            with pytest.raises(HivisError) as e:
                call(s, *args)
            assert e.value.code == HIVIS_EINVAL
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    good = dict(keep=i(2), add=i(2), held=i(2), table=i(2, 3), free_list=i(5), row_start=i(3), slots=i(4), positions=i(4), status=i(2))
    for name, t in (("keep", i(3)), ("held", torch.zeros(2)), ("table", i(6)), ("free_list", i(4)), ("row_start", i(2)), ("positions", i(5)), ("status", i(4)[::2])):
        with pytest.raises(HivisError):
            binding.kv4_plan(**dict(good, **{name: t}), block_tokens=16, n_blocks=4)
    q = torch.zeros(2, 4, 64)
    ok = dict(table=i(1, 2), row_start=i(2), kv_len=i(1), q=q, out=q.clone(), workspace=pool, mask=None)
    for name, t in (("table", i(2)), ("row_start", i(1)), ("kv_len", i(2)), ("q", q[0]), ("q", q.double()), ("q", q.transpose(0, 1).contiguous().transpose(0, 1)), ("out", q[:1]), ("out", q.bfloat16()),
                    ("mask", i(2)), ("mask", torch.zeros(3, dtype=torch.int64)), ("workspace", pool.float())):
        with pytest.raises(HivisError):
            binding.kv4_attend(s, pool, **dict(ok, **{name: t}), max_rows=2, max_len=20)
    lg, f = torch.zeros(2, 10), lambda *n: torch.zeros(n)
    for kw in (dict(logits=lg[0]), dict(logits=lg.half()), dict(logits=lg.t()), dict(tokens=i(3, 1)), dict(tokens=i(2, 1).long()), dict(logprob=f(2)), dict(logprob=None), dict(entropy=f(3)),
               dict(top_ids=i(2, 2)), dict(top_ids=i(2, 2), top_logprobs=f(2, 3)), dict(workspace=f(100))):
        args = dict(dict(logits=lg, tokens=i(2, 1), logprob=f(2, 1), workspace=pool), **kw)
        with pytest.raises(HivisError):
            binding.logprobs(**args)
    assert np.isfinite(binding.logprobs_bytes(3, 100, 4))
