"""GPU parity of the engine with the target's cache in 8 bits (DEER_KV_E4M3) against the oracle's decoder with such a cache: prompts of
one and of several passes, decoding with rejected blocks, a pool of few pages, injected rows.

Tolerance of logits: that of the tiny shapes elsewhere (2e-3).  What 8 bits add: K and V rows are rounded to bf16 from values that
differ in the last fp32 digits, so that now and then a bf16, and with it an e4m3, falls to the other side.  A key element that is off
by a whole e4m3 step (2^-3 of it; K's elements are below 1, q's too) moves a score by less than 2^-3 / sqrt(32) = 0.02, one weight of
many by 2 % of itself, and a logit by less than that weight's share of the attention's contribution (logits are below 1): with 20 or
more keys visible behind a complete page, under 1e-3."""
import numpy as np
import pytest

import deer_inputs as di
from gpu_common import StoredWeights, gpu_available
from kv8_reference import PAGE, page_values
from oracle import deer_oracle as O

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


class Kv8Decoder(O.Decoder):
    """Rows read the pages before their own as 8 bits stand for them, their own page in bf16."""

    def forward(self, ids, pos, cache, allowed_new, keep, logits_rows=None):
        s, R, n0 = self.s, len(ids), cache.n
        h = self._w("embed")[np.asarray(ids)]
        ones = np.ones(s.d_model, dtype=self.dtype)
        total = n0 + R
        for l in range(s.n_layers):
            a = O.rmsnorm(h, ones, s.rms_eps)
            q = O.rope((a @ self._w("wq", l)).reshape(R, s.n_q_heads, s.head_dim), pos, s.rope_base)
            k = O.rope((a @ self._w("wk", l)).reshape(R, s.n_kv_heads, s.head_dim), pos, s.rope_base)
            v = (a @ self._w("wv", l)).reshape(R, s.n_kv_heads, s.head_dim)
            k16 = np.concatenate([cache.K[l, :n0], O.round_to_bf16(k)])
            v16 = np.concatenate([cache.V[l, :n0], O.round_to_bf16(v)])
            cold = lambda x: np.concatenate([page_values(x[p:p + PAGE]) for p in range(0, total // PAGE * PAGE, PAGE)] + [x[total // PAGE * PAGE:]])   # noqa: E731
            k8, v8 = cold(k16), cold(v16)
            o = np.zeros_like(q)
            at = 0
            while at < R:                                    # rows of one page at a time
                own = int(pos[at]) // PAGE * PAGE
                n = min(R - at, own + PAGE - int(pos[at]))
                top = own + PAGE if own + PAGE < total else total
                see = np.arange(top)[None] <= np.asarray(pos)[at:at + n, None]
                o[at:at + n] = O.gqa_attention(q[at:at + n], np.concatenate([k8[:own], k16[own:top]]), np.concatenate([v8[:own], v16[own:top]]), see)
                at += n
            h = h + o.reshape(R, -1) @ self._w("wo", l)
            h = h + self._ffn(O.rmsnorm(h, ones, s.rms_eps), l)
            cache.K[l, n0:n0 + keep], cache.V[l, n0:n0 + keep] = k16[n0:n0 + keep], v16[n0:n0 + keep]
        cache.n = n0 + keep
        rows = np.arange(R) if logits_rows is None else np.asarray(logits_rows)
        return O.rmsnorm(h[rows], ones, s.rms_eps) @ self._w("lm_head") if len(rows) else np.zeros((0, s.vocab))


def shapes(**kw):
    t = di.ModelShape(**{**dict(n_layers=2, d_model=128, n_q_heads=4, n_kv_heads=2, head_dim=32, d_ff=512, vocab=1024, rope_base=10000.0), **kw})
    return t, di.CONFIGS["tiny"]["drafter"]


def engine(t, d, batch, max_seq, k, pages=0, fmt=1):
    from paper_2512_15176_amd import DeerEngine, binding
    wt, wd = StoredWeights(t, di.TARGET_SEED, "bf16"), StoredWeights(d, di.DRAFTER_SEED, "bf16")
    e = DeerEngine(t, d, batch, max_seq, k, di.mask_token_id(t.vocab), keep_logits=True, kv_format=fmt, kv_pages=pages)
    e.load_model(binding.DEER_TARGET, t, wt.for_engine)
    e.load_model(binding.DEER_DRAFTER, d, wd.for_engine)
    return e, wt, wd


def _logits(e, rows):
    out = np.empty((e.batch, rows, e.target.vocab), np.float32)
    e._check(e.lib.deer_debug_get_logits(e.ctx, 0, out.ctypes.data, out.size))
    return out


def decode(e, t, wt, prompts, capacity, k, steps, rng, tol=2e-3, bonus=False):
    """Blocks of random drafts, of which a random number is taken over, against the oracle's target."""
    import torch
    dec = Kv8Decoder(t, wt.as_f32)
    caches, xs = [], [list(p) for p in prompts]
    for p in prompts:
        c = O.KVCache(t, capacity, np.float64)
        if len(p) > 1:
            dec.forward(p[:-1], np.arange(len(p) - 1), c, None, len(p) - 1, [])
        caches.append(c)
    n = k + int(bonus)
    for _ in range(steps):
        blocks = rng.integers(0, t.vocab, (len(xs), k))
        e.draft_block(k, 0.0, 0)
        e.verify_block(k, 0.0, torch.tensor(blocks, dtype=torch.int32, device="cuda"))
        z = _logits(e, n)
        take = []
        for b, c in enumerate(caches):
            j = len(xs[b])
            rows = [xs[b][-1]] + [int(v) for v in blocks[b][:n - 1]]
            want = dec.forward(rows, np.arange(j - 1, j - 1 + n), c, None, n)
            assert np.abs(z[b] - want).max() < tol, (b, j, np.abs(z[b] - want).max())
            m = int(rng.integers(1, n + 1))                  # m - 1 drafts and one more token
            got = [int(v) for v in blocks[b][:m - 1]] + [int(rng.integers(0, t.vocab))]
            take.append(got)
            c.truncate(j - 1 + m)
            xs[b] += got
        e.debug_force_commit(take)
    assert e.get_lengths().tolist() == [len(x) for x in xs]
    return xs


CASES = [   # target shape, prompt lengths, block
    (dict(), [1, 50, 64, 65, 200], 8),
    (dict(head_dim=64, n_q_heads=14, n_kv_heads=2, d_model=256), [130, 3], 17),
    (dict(head_dim=128, n_q_heads=8, n_kv_heads=2), [300], 32),
    (dict(n_layers=6), [70, 129], 16),
    (dict(n_experts=8, top_k=2, d_ff_expert=128), [100, 30, 64], 12),
]


@pytest.mark.parametrize("shape,lens,k", CASES)
def test_decoding_against_the_oracle(shape, lens, k):
    t, d = shapes(**shape)
    e, wt, _ = engine(t, d, len(lens), 512, k)
    rng = np.random.default_rng(sum(lens))
    prompts = [di.prompt_ids(t.vocab, n, seq=b) for b, n in enumerate(lens)]
    e.prefill(prompts)
    decode(e, t, wt, prompts, 512, k, 6, rng)
    prompts = [[int(v) for v in p[::-1]] for p in prompts[::-1]]   # other sequences take their place
    e.prefill(prompts)
    decode(e, t, wt, prompts, 512, k, 2, rng)
    e.close()


def test_a_prompt_of_several_passes_and_the_bonus_token():
    t, d = shapes(n_layers=1)
    e, wt, _ = engine(t, d, 2, 4736, 16)
    e.set_bonus_token(True)
    prompts = [di.prompt_ids(t.vocab, 95, seq=0), di.prompt_ids(t.vocab, 4500, seq=1)]
    e.prefill(prompts)                                       # 3 + 125 tiles, of which the last would be half a page
    decode(e, t, wt, prompts, 4736, 16, 3, np.random.default_rng(1), bonus=True)
    e.close()


def test_one_block_is_its_tokens_one_by_one():
    """The same tokens through blocks of 16 and of 1, and as a prompt: the caches read the same."""
    import torch
    t, d = shapes()
    e, _, _ = engine(t, d, 1, 512, 16)
    ids = [int(v) for v in di.prompt_ids(t.vocab, 150)]
    last = []
    for n0, k in ((50, 16), (50, 1), (140, 1)):
        e.prefill([ids[:n0]])
        x = n0
        while x < 150 - k:
            e.draft_block(k)
            block = ids[x:x + k]
            e.verify_block(k, 0.0, torch.tensor([block], dtype=torch.int32, device="cuda"))
            z = e.debug_get_logits(0, k)[0]
            e.debug_force_commit([block])
            x += k
        e.draft_block(1)
        e.verify_block(1, 0.0, torch.tensor([[0]], dtype=torch.int32, device="cuda"))
        z1 = e.debug_get_logits(0, 1)[0]
        e.debug_force_commit([[]])
        last.append((x, z1, z))
    assert last[1][0] == last[2][0] and np.abs(last[1][1] - last[2][1]).max() < 1e-3
    assert last[0][0] == 146 and last[1][0] == 149
    e.close()


def test_eight_bits_are_near_bf16_and_not_the_same():
    import torch
    t, d = shapes()
    z = []
    for fmt in (0, 1):
        e, _, _ = engine(t, d, 1, 512, 8, fmt=fmt)
        e.prefill([di.prompt_ids(t.vocab, 300)])
        dr = e.draft_block(8, 1.0, 3)
        e.verify_block(8, 1.0, torch.arange(8, dtype=torch.int32, device="cuda")[None])
        z.append(e.debug_get_logits(0, 8)[0])
        acc, com, n = e.accept_and_commit(8, 1.0, 3)
        assert dr.shape == (1, 8) and 1 <= n[0] <= 8
        e.close()
    assert 0 < np.abs(z[0] - z[1]).max() < 2e-2


def test_a_pool_of_few_pages():
    from paper_2512_15176_amd import DeerError
    t, d = shapes()
    e, wt, _ = engine(t, d, 4, 512, 16, pages=8)
    rng = np.random.default_rng(2)
    with pytest.raises(DeerError) as err:
        e.prefill([di.prompt_ids(t.vocab, 200, seq=b) for b in range(3)])   # 12 pages
    assert err.value.status == -3
    prompts = [di.prompt_ids(t.vocab, n, seq=n) for n in (130, 60, 64)]     # 3 + 1 + 1
    e.prefill(prompts)
    decode(e, t, wt, prompts, 512, 16, 3, rng)
    for _ in range(40):                                      # until the block does not fit
        try:
            e.draft_block(16)
        except DeerError as err:
            assert err.status == -3
            break
        import torch
        e.verify_block(16, 0.0, torch.zeros(3, 16, dtype=torch.int32, device="cuda"))
        e.debug_force_commit([[1] * 16] * 3)
    else:
        raise AssertionError("the pool never ran out")
    prompts = [di.prompt_ids(t.vocab, 480, seq=7)]           # one long sequence takes every page
    e.prefill(prompts)
    decode(e, t, wt, prompts, 512, 16, 1, rng)
    e.close()


def test_injected_rows():
    import torch
    from paper_2512_15176_amd import DeerError
    t, d = shapes()
    e, wt, _ = engine(t, d, 2, 8192, 8)
    rng = np.random.default_rng(3)
    dec = Kv8Decoder(t, wt.as_f32)
    lens = [6000, 77]                                        # more than a pass's rows; part of a page
    caches = [O.KVCache(t, 8192, np.float64) for _ in lens]
    for l in range(t.n_layers):
        for b, n in enumerate(lens):
            kb, vb = (di.kv_fill_bits(t, w, l, b, n) for w in "kv")
            e.debug_load_kv(0, l, b, 0, torch.from_numpy(kb.view(np.int16)).cuda(), torch.from_numpy(vb.view(np.int16)).cuda())
            caches[b].K[l, :n], caches[b].V[l, :n] = di.bf16_bits_to_f32(kb), di.bf16_bits_to_f32(vb)
            caches[b].n = n
    for bad in ([6002, 78], [30, 78]):                       # not loaded; a page that is in 8 bits only
        with pytest.raises(DeerError):
            e.set_prefilled(bad, [1, 2])
    e.set_prefilled([6001, 78], [5, 9])
    e.draft_block(8)
    block = rng.integers(0, t.vocab, (2, 8))
    e.verify_block(8, 0.0, torch.tensor(block, dtype=torch.int32, device="cuda"))
    z = e.debug_get_logits(0, 8)
    for b, last in enumerate((5, 9)):
        want = dec.forward([last] + [int(v) for v in block[b][:7]], np.arange(lens[b], lens[b] + 8), caches[b], None, 8)
        assert np.abs(z[b] - want).max() < 2e-3
    with pytest.raises(DeerError):
        e.get_kv_layout(0)
    assert e.get_kv_layout(1).head_dim == d.head_dim
    e.close()
