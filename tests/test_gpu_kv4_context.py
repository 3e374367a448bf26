"""Contexts whose target cache is held in 4 bits (hivis_create_kv4), and log probabilities of a context's rows.

The oracle follows what the library holds: after every pass the new rows of every layer are read back with hivis_kv4_get, each value has to be within
half a step of the format of the oracle's own key or value, and the oracle then goes on with the held ones.  Everything else (features, logits, tokens,
lengths, trees) is compared as for ordinary contexts, with the same tolerances."""
import numpy as np
import pytest

import operator_reference as ref
import parity_utils
import synth
import test_gpu_tree
from oracle import HivisOracle
from oracle.model import KVCache
from oracle.tree import HivisTreeOracle
from paper_2509_23928_amd import HIVIS_ECAP, HIVIS_EINVAL, HIVIS_ESTATE, Hivis, HivisError
from test_gpu_parity import small_bf16

pytestmark = pytest.mark.gpu


class HeldHivis(Hivis):
    """Reads back what every pass left in the target cache."""
    def _record(self, first, n):
        self.held = {(b, l): (int(first[b]),) + self.kv4_get(l, b, int(first[b]), n) for b in range(self.B) for l in range(self.cfg.n_layers)}

    def prefill(self, vis, ids):
        first = super().prefill(vis, ids)
        self._record([0] * self.B, vis.shape[-2] + ids.shape[-1])
        return first

    def verify(self):
        super().verify()
        self._record(self.kv_lengths()[0], self.K + 1)

    def tree_verify(self):
        super().tree_verify()
        self._record(self.kv_lengths()[0], self.tree_shape[2] + 1)


class HeldCache(KVCache):
    def __init__(self, cfg, hv, seq, layer):
        super().__init__(cfg.n_kv_heads, cfg.head_dim)
        self.hv, self.at, self.loose = hv, (seq, layer), 1e-3 if cfg.dtype == "f32" else 3e-2

    def append(self, k, v, pos):
        first, hk, hv = self.hv.held[self.at]
        assert first == len(self) and hk.shape == k.shape
        for mine, held in ((k, hk), (v, hv)):
            delta = self.loose * np.sqrt(np.mean(mine ** 2))                    # what the passes before may differ by
            # (a key's dims lie pair by pair in the cache)
            pairs = (lambda x: np.stack(np.split(x, 2, -1), -1)) if mine is k else (lambda x: x)
            g, h = (pairs(x.astype(np.float64)).reshape(-1, 32) for x in (mine, held))
            m, e = np.frexp(np.abs(g).max(-1) + delta)
            s = np.exp2(np.where(2 * m <= 1.75, e - 3, e - 2))[:, None]
            y = np.maximum(np.abs(g), np.abs(h)) / s
            assert (np.abs(g - h) <= s * np.where(y < 2, 0.25, np.where(y < 4, 0.5, 1.0)) + delta).all()
        super().append(hk.astype(np.float64), hv.astype(np.float64), pos)


def following(base, hv):
    """A class of oracles that follow hv, one per sequence."""
    class Oracle(base):
        count = 0

        def __init__(self, cfg, weights):
            super().__init__(cfg, weights)
            self.target.caches = [HeldCache(cfg, hv, Oracle.count, l) for l in range(cfg.n_layers)]
            Oracle.count += 1
    return Oracle


CONFIGS = {
    "tiny fp32": lambda: synth.get_config("C1"),
    "fp32, two sequences": lambda: synth.get_config("C1").scaled(batch=2, K=3, n_vis=33, n_text=20),
    "fp32 phases off": lambda: synth.get_config("C1").scaled(batch=4, K=7, n_vis=40, n_text=9),
    "bf16 heads of 128": lambda: small_bf16(),
    "bf16 grouped": lambda: small_bf16(n_q_heads=7, n_kv_heads=1, d=896, ffn=2368, K=6, n_vis=200, n_text=70, rope_theta=1e6, rms_eps=1e-6),
    "bf16 heads of 64": lambda: small_bf16(n_q_heads=8, n_kv_heads=4, head_dim=64, K=3),
    "bf16 four sequences": lambda: small_bf16(batch=4, K=7, n_vis=90, n_text=45),
    "bf16 two sequences, twelve rows": lambda: small_bf16(batch=2, K=5, n_vis=70, n_text=30),
    "bf16 no visual rows, short prompt": lambda: small_bf16(n_vis=0, n_text=6, K=2),
    "bf16 long prompt": lambda: small_bf16(n_vis=700, n_text=60, d=256, n_q_heads=2, n_kv_heads=2, ffn=512, vocab=1024, K=4),
}


@pytest.mark.parametrize("name,block", [(n, b) for i, n in enumerate(CONFIGS) for b in ((16, 64) if i in (0, 3) else ((32, 256, 16, 128)[i % 4],))])
def test_cycles(monkeypatch, name, block):
    cfg = CONFIGS[name]()
    w = synth.make_weights(cfg, seed=3)
    vis, ids = synth.make_prompt(cfg, seed=3)
    hv = HeldHivis(cfg, w, kv4_block=block)
    monkeypatch.setattr(parity_utils, "HivisOracle", following(HivisOracle, hv))
    sbs = parity_utils.SideBySide(cfg, w, hv, vis, ids)
    for _ in range(4):
        sbs.cycle(cfg.K)
    hv.close()
    print(name, block, sbs.summary())


@pytest.mark.parametrize("switch", ["HIVIS_FUSED=0", "HIVIS_ATTN_ELECT=0", "HIVIS_WIDE_GEMM=0", "HIVIS_ATTN_SHARED_MIN=8"])
@pytest.mark.parametrize("name", ["bf16 four sequences", "bf16 no visual rows, short prompt"])
def test_cycles_under_switches(monkeypatch, name, switch):
    monkeypatch.setenv(*switch.split("="))
    cfg = CONFIGS[name]()
    w = synth.make_weights(cfg, seed=4)
    vis, ids = synth.make_prompt(cfg, seed=4)
    hv = HeldHivis(cfg, w, kv4_block=32)
    monkeypatch.setattr(parity_utils, "HivisOracle", following(HivisOracle, hv))
    sbs = parity_utils.SideBySide(cfg, w, hv, vis, ids)
    for _ in range(3):
        sbs.cycle(cfg.K)
    hv.close()


def test_one_launch_per_pass_is_refused(monkeypatch):
    monkeypatch.setenv("HIVIS_PERSISTENT", "1")
    cfg = small_bf16()
    with pytest.raises(HivisError) as e:
        Hivis(cfg, synth.make_weights(cfg, seed=4), kv4_block=32)
    assert e.value.code == HIVIS_EINVAL and "HIVIS_PERSISTENT" in str(e.value)


def test_accepted_drafts_move_the_lengths(monkeypatch):
    """Drafts that the target accepts: sequences of a batch grow apart, and rows of rejected drafts give their places back."""
    cfg = small_bf16(batch=3, K=4, n_vis=20, n_text=11)
    w = synth.make_weights(cfg, seed=5)
    vis, ids = synth.make_prompt(cfg, seed=5)
    scout = Hivis(cfg, w, kv4_block=16)
    first = scout.prefill(vis, ids)
    line = [[int(first[b])] for b in range(cfg.batch)]
    for _ in range(9):                                                         # what the target says, a token at a time
        scout.set_drafts([[0]] * cfg.batch)
        scout.verify()
        t = scout.get_tokens()[1]
        n, tok = scout.accept()
        for b in range(cfg.batch):
            line[b] += [int(x) for x in tok[b, :n[b] + 1]]
        assert t.shape == (cfg.batch, 2)
    scout.close()
    hv = HeldHivis(cfg, w, kv4_block=16)
    monkeypatch.setattr(parity_utils, "HivisOracle", following(HivisOracle, hv))
    sbs = parity_utils.SideBySide(cfg, w, hv, vis, ids)
    accepted = [0] * cfg.batch
    for cycle in range(3):
        drafts = []
        for b in range(cfg.batch):
            nxt = line[b][len(sbs.emitted[b]):][:cfg.K]
            good = (cycle + 2 * b) % (cfg.K + 1) if sbs.emitted[b] == line[b][:len(sbs.emitted[b])] else 0
            drafts.append([t if i < good else (t + 1) % cfg.vocab for i, t in enumerate(nxt + [0] * (cfg.K - len(nxt)))])
        for b, o in enumerate(sbs.cycle(cfg.K, drafts)):
            accepted[b] += o["n"]
    assert len(set(hv.kv_lengths()[0].tolist())) > 1 and sum(accepted) > 4, accepted
    hv.close()


@pytest.mark.parametrize("name", ["tiny fp32", "bf16 heads of 128", "bf16 grouped"])
def test_trees(monkeypatch, name):
    cfg = CONFIGS[name]()
    def make(cfg, seed, room):
        w = synth.make_weights(cfg, seed=seed)
        vis, ids = synth.make_prompt(cfg, seed=seed)
        hv = HeldHivis(cfg, w, max_text=cfg.n_text + room, k_max=max(cfg.K, 1), kv4_block=16)
        monkeypatch.setattr(test_gpu_tree, "HivisTreeOracle", following(HivisTreeOracle, hv))
        return w, vis, ids, hv
    monkeypatch.setattr(test_gpu_tree, "make_tree", make)
    t = test_gpu_tree.TreeSideBySide(cfg, 2)
    for shape in ((4, 3, 10), (2, 2, 4), (6, 3, 30)):
        t.cycle(*shape)
    t.hv.close()


@pytest.mark.parametrize("name", ["tiny fp32", "bf16 heads of 128"])
def test_the_path_of_a_tree_moves_next_to_the_root(name):
    """Root -> (wrong, right) -> (wrong, right) and a right third: the followed rows 2, 4, 5 move to 1, 2, 3, bit for bit, in every layer."""
    cfg = CONFIGS[name]()
    w = synth.make_weights(cfg, seed=4)
    vis, ids = synth.make_prompt(cfg, seed=4)
    scout = Hivis(cfg, w, kv4_block=16)
    line = [int(scout.prefill(vis, ids)[0])]
    for _ in range(3):
        scout.set_drafts([[0] * 1])
        scout.verify()
        n, tok = scout.accept()
        line += [int(x) for x in tok[0, :n[0] + 1]]
    scout.close()
    hv = Hivis(cfg, w, kv4_block=16)
    assert int(hv.prefill(vis, ids)[0]) == line[0]
    wrong = [(t + 1) % cfg.vocab for t in line]
    hv.tree_set([wrong[1], line[1], wrong[2], line[2], line[3]], [0, 0, 2, 2, 4])
    base = int(hv.kv_lengths()[0][0])
    hv.tree_verify()
    before = [hv.kv4_get(l, 0, base, 6) for l in range(cfg.n_layers)]
    n, tok = hv.tree_accept()
    assert n == 3 and [int(t) for t in tok[:3]] == line[1:4]
    assert int(hv.kv_lengths()[0][0]) == base + 4
    for l in range(cfg.n_layers):
        for was, now in zip(before[l], hv.kv4_get(l, 0, base, 4)):
            np.testing.assert_array_equal(now, was[[0, 2, 4, 5]])
    hv.close()


def test_pool_of_blocks():
    """A pool smaller than all sequences could fill: calls that would need more return ECAP and change nothing; a new prompt takes the blocks again."""
    cfg = synth.get_config("C1").scaled(batch=2, K=4, n_vis=20, n_text=12)
    w = synth.make_weights(cfg, seed=1)
    vis, ids = synth.make_prompt(cfg, seed=1)
    hv = Hivis(cfg, w, kv4_block=16, kv4_blocks=6)                             # 48 rows each
    for _ in range(2):
        hv.prefill(vis, ids)                                                   # 32 rows: two blocks each
        cycles = 0
        while True:
            before = hv.kv_lengths()
            try:
                hv.set_drafts([[0] * 4] * 2)
            except HivisError as e:
                assert e.code == HIVIS_ECAP and "blocks" in str(e)
                break
            hv.verify()
            hv.accept()
            cycles += 1
        assert max(before[0]) + 5 > 48 and cycles >= 2
        after = hv.kv_lengths()
        assert all((a == b).all() for a, b in zip(before, after))
        if max(before[0]) + 2 <= 48:
            hv.set_drafts([[0]] * 2)
    with pytest.raises(HivisError) as e:
        Hivis(cfg, w, kv4_block=16, kv4_blocks=2).prefill(vis, ids)
    assert e.value.code == HIVIS_ECAP
    hv.close()


def test_refusals():
    cfg = synth.get_config("C1")
    w = synth.make_weights(cfg, seed=1)
    vis, ids = synth.make_prompt(cfg, seed=1)
    for block, blocks in ((8, 0), (24, 0), (512, 0), (0, 0), (-16, 0), (16, -1)):
        with pytest.raises(HivisError) as e:
            Hivis(cfg, w, kv4_block=block, kv4_blocks=blocks)
        assert e.value.code == HIVIS_EINVAL
    hv = Hivis(cfg, w, kv4_block=16)
    for call in (lambda: hv.kv4_get(0, 0, 0, 1), lambda: hv.get_logprobs(2)):
        with pytest.raises(HivisError) as e:
            call()
        assert e.value.code == HIVIS_ESTATE
    hv.prefill(vis, ids)
    for args in ((-1, 0, 0, 1), (cfg.n_layers, 0, 0, 1), (0, 1, 0, 1), (0, 0, -1, 1), (0, 0, 96, 1), (0, 0, 0, 97), (0, 0, 5, -1)):
        with pytest.raises(HivisError) as e:
            hv.kv4_get(args[0], args[1], args[2], args[3]) if args[3] >= 0 else hv._check(hv.lib.hivis_kv4_get(hv.ctx, *args, 0x1000, 0x1000))
        assert e.value.code == HIVIS_EINVAL
    assert hv.kv4_get(0, 0, 96, 0)[0].shape[0] == 0
    for kw in (dict(temperature=0.0), dict(temperature=float("nan")), dict(top_k=33), dict(tokens=[[0] * 65])):
        with pytest.raises(HivisError) as e:
            hv.get_logprobs(2, **kw)
        assert e.value.code == HIVIS_EINVAL
    hv.close()
    plain = Hivis(cfg, w)
    plain.prefill(vis, ids)
    with pytest.raises(HivisError) as e:
        plain.kv4_get(0, 0, 0, 1)
    assert e.value.code == HIVIS_ESTATE
    plain.close()


@pytest.mark.parametrize("kv4", [None, 16])
@pytest.mark.parametrize("name", ["fp32, two sequences", "bf16 heads of 128"])
def test_logprobs_of_the_rows(name, kv4):
    """Of the prompt's last row, a draft round and a verify pass (chain and tree), against the logits that get_logits returns."""
    cfg = CONFIGS[name]()
    w = synth.make_weights(cfg, seed=2)
    vis, ids = synth.make_prompt(cfg, seed=2)
    hv = Hivis(cfg, w, kv4_block=kv4)

    def check(which, tokens, T=1.0, top=4):
        x = hv.get_logits(which).astype(np.float64).reshape(-1, cfg.vocab)
        got = hv.get_logprobs(which, tokens, temperature=T, top_k=top)
        want = ref.logprobs(x, np.asarray(tokens).reshape(len(x), -1), T, top)
        tol = 2.0 ** -24 * (8 * (np.ptp(x) / T + 1) + cfg.vocab / 16 + 64)
        np.testing.assert_allclose(got[0], want[0], rtol=2.0 ** -22, atol=tol)
        np.testing.assert_allclose(got[1], want[1], rtol=2.0 ** -22, atol=2 * tol * (1 + np.log(cfg.vocab)))
        np.testing.assert_array_equal(got[2], want[2])
        np.testing.assert_allclose(got[3], want[3], rtol=2.0 ** -22, atol=tol)

    B, K = cfg.batch, cfg.K
    first = hv.prefill(vis, ids)
    check(2, first[:, None])
    hv.draft(K)
    hv.verify()
    drafts, target = hv.get_tokens()
    check(1, drafts.T.reshape(-1, 1), T=0.8)
    check(0, np.stack([target.reshape(-1), target.reshape(-1) // 2], 1), top=32)
    hv.accept()
    check(0, target.reshape(-1, 1), T=1.7, top=1)
    lp = hv.get_logprobs(0)
    assert lp[0].shape == (B * (K + 1), 0) and np.isfinite(lp[1]).all()
    if B == 1:
        hv.tree_draft(3, 2, 7)
        hv.tree_verify()
        x = hv.tree_get(verified=True)["target_tokens"]
        check(0, x[:, None])
    hv.close()
