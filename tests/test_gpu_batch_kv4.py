"""Batched decoding over a paged cache held in 4 bits: what a prompt and a step leave in the pages is the quantised form of what
they leave in 16 bits, and a step's logits are those of the model that attends over exactly these values (the oracle's operators
in 64 bits, layer by layer, on the cache as the library reads it back)."""
import numpy as np
import pytest
import torch

import kv4_utils as ku
from paper_2604_23467_amd import workloads as wl
from parity_utils import check_greedy_token, check_logits

pytestmark = pytest.mark.gpu


def _session(cfg, w_np, flags=0):
    from paper_2604_23467_amd import binding
    assert torch.cuda.is_available(), "these tests need a GPU"
    return binding.Session(cfg, wl.weights_to_torch(w_np, device="cuda:0", dtype=torch.float16), flags=flags)


def held(x, cfg):
    """Rows [n, d_model] as the cache holds and reads them: (values, steps)"""
    x = torch.from_numpy(np.ascontiguousarray(x)).reshape(x.shape[0], cfg["n_heads"], cfg["head_dim"])
    c, s, mid = ku.quantise(x)
    return ku.values(c, s, mid).reshape(x.shape[0], -1).numpy(), s.repeat_interleave(32, -1).reshape(x.shape[0], -1).numpy()


def model_step(o, cfg, w, token, cache):
    """Logits of the model at the last position of `cache` (per layer K and V [positions, d_model], the newest included), and the
    newest keys and values that each layer computes."""
    d, H, hd = cfg["d_model"], cfg["n_heads"], cfg["head_dim"]
    pos = cache[0][0].shape[0] - 1
    x, new = np.asarray(w["tok_emb"][token], dtype=np.float64), []
    for L, (K, V) in zip(w["layers"], cache):
        a = o.rmsnorm(x, L["attn_norm"], cfg["rms_eps"])
        q = o.rope(o.matvec(L["wq"], a), H, hd, pos, cfg["rope_theta"])
        new.append((o.rope(o.matvec(L["wk"], a), H, hd, pos, cfg["rope_theta"]), o.matvec(L["wv"], a)))
        out = np.concatenate([o.attention_head(q[h * hd:(h + 1) * hd], K[:, h * hd:(h + 1) * hd], V[:, h * hd:(h + 1) * hd])[0] for h in range(H)])
        x = x + o.matvec(L["wo"], out)
        a = o.rmsnorm(x, L["ffn_norm"], cfg["rms_eps"])
        x = x + o.matvec(L["w_down"], o.swiglu(o.matvec(L["w_gate"], a), o.matvec(L["w_up"], a)))
    return o.matvec(w["lm_head"], o.rmsnorm(x, w["final_norm"], cfg["rms_eps"])), new


@pytest.mark.parametrize("heads,head_dim,page,slots,flags", [(4, 64, 8, 4, 0), (4, 64, 16, 20, 0), (2, 128, 16, 4, 0), (2, 128, 5, 17, 1),
                                                             (3, 64, 16, 3, 32)])
def test_steps_over_a_cache_in_4_bits(oracle64, heads, head_dim, page, slots, flags):
    """Sequences of several lengths, over page borders and over the tiles' (32 keys), joining and leaving."""
    cfg = wl.custom_cfg(2, heads, head_dim, 688, 512, 400)
    w = wl.weights_astype(wl.make_weights_numpy(cfg, seed=3), np.float16)
    lens = (1, 31, 40, 300)[:min(slots, 4)]
    prompts = [wl.make_tokens(n, cfg["vocab"], seed=50 + n) for n in lens]
    rows16 = []
    with _session(cfg, w, flags) as s:
        s.ll_batch_open(slots, page, sum(n // page + 4 for n in lens) + 1)
        for p in prompts:
            slot, _ = s.ll_batch_add(p)
            rows16.append([[s.ll_batch_dbg_get_kv(slot, l, k, len(p)) for k in range(2)] for l in range(2)])
        s.ll_batch_close()
        s.ll_batch_open(slots, page, sum(n // page + 4 for n in lens) + 1, kv_bits=4)
        live = {}
        for i, p in enumerate(prompts):
            slot, t = s.ll_batch_add(p)
            live[slot] = [t, len(p)]
            for l in range(2):
                for k in range(2):
                    want = held(rows16[i][l][k], cfg)[0]
                    got = s.ll_batch_dbg_get_kv(slot, l, k, len(p))
                    assert (np.abs(got - want) <= 2.0 ** -10 * np.abs(want) + 2.0 ** -25).all(), (i, l, k)
        for step in range(6):
            if step == 3:                                        # one leaves, its pages serve a newcomer
                gone = sorted(live)[0]
                s.ll_batch_remove(gone)
                del live[gone]
                slot, t = s.ll_batch_add(prompts[-1][:37])
                assert slot == gone
                live[slot] = [t, 37 if len(prompts[-1]) >= 37 else len(prompts[-1])]
            toks = s.ll_batch_step()
            assert all((t >= 0) == (b in live) for b, t in enumerate(toks)), toks
            for b, (fed, n) in live.items():
                cache = [[s.ll_batch_dbg_get_kv(b, l, k, n + 1).astype(np.float64) for k in range(2)] for l in range(2)]
                logits, new = model_step(oracle64, cfg, w, fed, cache)
                got = s.ll_batch_dbg_get_logits(b)
                what = "slot %d step %d" % (b, step)
                check_logits(got, logits, what)
                check_greedy_token(toks[b], got, what)
                for l in range(2):                               # the newest row is its own quantised form
                    for k in range(2):
                        _, st = held(new[l][k][None], cfg)
                        off = np.abs(cache[l][k][-1] - new[l][k])
                        assert (off <= 0.5 * 1.02 * st[0] + 2e-2 * np.sqrt(np.mean(new[l][k] ** 2))).all(), (what, l, k)
                live[b] = [toks[b], n + 1]
        s.ll_batch_close()
        assert s.ll_reset() == 0 and s.ll_prefill(prompts[0]) >= 0 and s.ll_decode_step() >= 0


def test_4_bits_take_less_than_a_third_of_the_pool():
    from paper_2604_23467_amd import binding as b
    cfg = wl.custom_cfg(2, 4, 128, 688, 512, 400)
    with _session(cfg, wl.make_weights_numpy(cfg, seed=3)) as s:
        many = 4000
        full, small = (s.lib.ll_batch_pool_bytes_kv(16, many, bits) for bits in (16, 4))
        assert s.lib.ll_batch_pool_bytes(16, many) == full
        assert small < full / 3
        for bits in (0, 8, 5, -4):
            assert s.lib.ll_batch_pool_bytes_kv(16, many, bits) == 0
        assert s.lib.ll_batch_pool_bytes_kv(1 << 13, (1 << 13) + 1, 4) == 0
        import ctypes as C
        assert s.lib.ll_batch_open_kv(4, 16, many, 8, C.c_void_p(256), small) == b.LL_E_BAD_ARG
        assert s.lib.ll_batch_open_kv(4, 1 << 13, (1 << 13) + 1, 4, C.c_void_p(256), 1 << 45) == b.LL_E_BAD_ARG
        pool = torch.empty(small + 256, dtype=torch.uint8, device="cuda:0")
        at = (pool.data_ptr() + 255) // 256 * 256
        assert s.lib.ll_batch_open_kv(4, 16, many, 4, C.c_void_p(at), small // 2) == b.LL_E_WORKSPACE
        assert s.lib.ll_batch_open_kv(4, 16, many, 4, C.c_void_p(at + 16), small) == b.LL_E_WORKSPACE
        assert s.lib.ll_batch_open_kv(4, 16, many, 4, C.c_void_p(at), small) == b.LL_OK
        slot, _ = s.ll_batch_add([1, 2, 3])
        out = (C.c_float * (4 * cfg["d_model"]))()
        for args in ((slot, 2, 0, 1), (slot, 0, 2, 1), (slot, 0, 0, 4), (slot + 1, 0, 0, 1), (slot, -1, 0, 1), (slot, 0, 0, -1)):
            assert s.lib.ll_batch_dbg_get_kv(*args, out) == b.LL_E_BAD_ARG
        assert s.lib.ll_batch_dbg_get_kv(slot, 0, 0, 3, out) == b.LL_OK


@pytest.mark.parametrize("slots", [4, 32])
def test_graph_and_eager_steps_give_the_same_bits(slots):
    """... and the same as themselves, with free slots between the sequences and lengths that are cut into shares."""
    cfg = wl.custom_cfg(1, 4, 128, 1024, 512, 2100)
    w = wl.make_weights_numpy(cfg, seed=9)
    prompts = [wl.make_tokens(n, cfg["vocab"], seed=n) for n in (3, 2000, 64, 700)]

    def run(flags):
        out = []
        with _session(cfg, w, flags) as s:
            s.ll_batch_open(slots, 16, 260, kv_bits=4)
            for p in prompts:
                s.ll_batch_add(p)
            s.ll_batch_remove(2)
            for _ in range(5):
                toks = s.ll_batch_step()
                out.append((toks, [s.ll_batch_dbg_get_logits(b).copy() for b in (0, 1, 3)]))
            assert 0.0 < s.ll_batch_dbg_time_steps(3)
            out.append((s.ll_batch_step(), [s.ll_batch_dbg_get_logits(b).copy() for b in (0, 1, 3)]))
        return out
    first = run(0)
    for other in (run(0), run(1)):
        for (ta, la), (tb, lb) in zip(first, other):
            assert ta == tb
            assert all(np.array_equal(x, y) for x, y in zip(la, lb))


def test_sampling_and_capacity_in_4_bits():
    from paper_2604_23467_amd import binding as b
    cfg = wl.tiny_cfg(max_seq=64)
    with _session(cfg, wl.make_weights_numpy(cfg, seed=2)) as s:
        s.ll_set_sampling(0.8, top_k=20, top_p=0.9, seed=5)
        s.ll_batch_open(3, 4, 8, kv_bits=4)
        s.ll_batch_add(wl.make_tokens(9, cfg["vocab"], seed=1))            # 3 of 7 pages
        s.ll_batch_add(wl.make_tokens(11, cfg["vocab"], seed=2))           # 3
        with pytest.raises(b.LLError) as e:
            s.ll_batch_add(wl.make_tokens(8, cfg["vocab"], seed=3))
        assert e.value.code == b.LL_E_CAPACITY
        assert all(0 <= t < cfg["vocab"] for t in s.ll_batch_step()[:2])   # the second takes the last page
        with pytest.raises(b.LLError) as e:
            for _ in range(8):
                s.ll_batch_step()
        assert e.value.code == b.LL_E_CAPACITY
