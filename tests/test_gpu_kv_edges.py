"""Calls of the paged cache at the ends of what its documentation allows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import kv as ok
from tests.test_gpu_kv import DEV, Pool, attn_bound, bd_, dev, host, run_attention, small_model

pytestmark = pytest.mark.gpu


def test_pages_with_the_largest_slot_map():
    """A map of 2^31 - 1 rows, the most that its argument holds, of which 40 are written."""
    bd = bd_()
    cap = 2 ** 31 - 1
    if torch.cuda.mem_get_info(DEV)[0] < 48 << 30:
        pytest.skip("needs 34 GB")
    i32 = torch.empty(2 * cap, dtype=torch.int32, device=DEV)
    slot = torch.empty(cap, dtype=torch.int64, device=DEV)
    i32[40], slot[40] = -5, -6
    table, free = dev([[-1, -1]]), dev(np.arange(8))
    have, want, count, info, start = dev([0]), dev([40]), dev([8]), dev([0, 0, 0, 0]), dev([0, 0])
    bd.bd_kv_pages(1, 32, 2, 8, have.data_ptr(), want.data_ptr(), table.data_ptr(), free.data_ptr(), count.data_ptr(), info.data_ptr(),
                   cap, start.data_ptr(), i32.data_ptr(), i32[cap:].data_ptr(), slot.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert host(info).tolist() == [6, 40, 0, 2] and host(table).tolist() == [[7, 6]]
    assert host(slot[:40]).tolist() == [7 * 32 + i for i in range(32)] + [6 * 32 + i for i in range(8)]
    assert host(i32[cap:cap + 40]).tolist() == list(range(40)) and int(i32[40]) == -5 and int(slot[40]) == -6


def test_requests_that_are_left_out():
    """A negative first row or position leaves the request out, whatever its other rows; the requests beside it are served."""
    bd = bd_()
    H, hd, T = 2, 64, 32
    pool = Pool(370, 8, H, hd, T)
    cache = pool.cache()
    table = np.array([[0, 1], [2, 3], [4, 5]], dtype=np.int32)
    x = dev(pool.rng.standard_normal((50, H, hd)), torch.float32)
    before = [host(t) for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    for start, pos0 in (([-4, 20, 20, 20], [0, 0, 0]), ([0, 20, 20, 20], [-5, 0, 0])):
        bd.kv_store(cache, x, x, dev(table), dev(start), dev(pos0))
        assert all((a == host(t)).all() for a, t in zip(before, (cache.k, cache.v, cache.k_scale, cache.v_scale)))
        out = torch.full_like(x, 3.0)
        bd.kv_read(cache, dev(table), dev(start), dev(pos0), out, out.clone())
        assert (host(out) == 3.0).all()
    start, pos0 = [-3, 20, 30, 50], [0, -2, 40]
    out, q = torch.full_like(x, 3.0), dev(pool.rng.standard_normal((50, 4, hd)), torch.float32)
    bd.kv_read(cache, dev(table), dev(start), dev(pos0), out, torch.empty_like(out))
    want, _ = ok.cached(pool.kc, pool.ks, table[2], 60)
    assert (host(out)[:30] == 3.0).all() and (host(out)[30:] == want[40:]).all()
    # the attention serves rows at positions from 0 on; rows before them are zeros
    o = bd.kv_attention(cache, q, dev(table), dev(start), dev(pos0), dev([64, 64, 60]), 1, out=torch.full_like(q, 3.0))
    ref, mag, big = ok.attention(pool.kc, pool.ks, pool.vc, pool.vs, host(q), table, [20, 20, 30, 50], pos0, [64, 64, 60], 1)
    bound = attn_bound(ref, mag, big, hd, 64, torch.float32)
    assert (host(o)[:20] == 3.0).all() and (host(o)[20:22] == 0).all()
    assert (np.abs(host(o) - ref)[20:] <= bound[20:]).all() and (host(o)[22:] != 0).any()


@pytest.mark.parametrize("kw", [{}, dict(n_experts=8, top_k=2, expert_ffn=128, n_shared=1, ffn_dim=0)])
def test_memory_of_states(kw):
    """What a state of 8-bit pages takes less than one of pairs is what the sweep counts, workspaces of either left out (and
    the caches' memory is a quarter: the rows before they are coded take none of their own)."""
    from paper_2609_33887_amd.sweep import cache_bytes
    bd = bd_()
    w, ws, prompts = small_model(n_layers=4, d_model=512, n_heads=8, n_kv_heads=4, head_dim=128, batch=8, prompt_len=2048, gen_len=64,
                                 **dict(dict(ffn_dim=1024), **kw))
    took = {}
    for kv in (None, "fp8"):
        m = bd.Model(w, ws, DEV, kv=kv)
        torch.cuda.synchronize()
        free = torch.cuda.mem_get_info(DEV)[0]
        st = bd.State(m, prompts, w.gen_len, 0.9, 2, 16)
        torch.cuda.synchronize()
        took[kv] = free - torch.cuda.mem_get_info(DEV)[0]
        st.close()
        m.close()
    want = cache_bytes(w) - cache_bytes(w, "fp8")
    work = bd.bd_kv_attention_workspace(8, 4, 128, 8, 512, 32, 32, 66)
    # a buffer's slack of 64 KB each, allocations in 2 MB
    assert want - work - (4 << 20) <= took[None] - took["fp8"] <= want + (24 << 20), (took, want, work)
    assert 3.9 * cache_bytes(w, "fp8") <= cache_bytes(w)


def test_profile_classes_of_a_coded_decode():
    """The attention class holds one launch a layer and step (the prompt's last layer has none), whichever the cache; the
    coding of K and V has a class of its own."""
    bd = bd_()
    w, ws, prompts = small_model()
    for kv in (None, "fp8"):
        m = bd.Model(w, ws, DEV, kv=kv)
        bd.bd_profile(m.handle, True)
        st = bd.State(m, prompts, w.gen_len, 0.9, 2, 16)
        for _ in range(3):
            st.step()
            st.commit()
        prof = bd.bd_profile_read(m.handle)
        st.close()
        m.close()
        assert prof["attn"][1] == 2 * 3 + 1 and prof["gemm_qkv"][1] == 2 * 4, prof
        assert prof["rope"][1] == (2 * 4 if kv else 0) and (prof["rope"][0] > 0) == bool(kv), prof


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd", [64, 128])
def test_cut_keys_of_the_most_requests(hd, dtype):
    """1024 requests, of which 40 have rows, one of them 5000 keys: the plan's sums over more requests than a workgroup has
    threads, requests from number 256 on, the most local memory, keys cut into ranges."""
    n, T = 1024, 32
    rng = np.random.default_rng([73, hd])
    at = [3, 255, 256, 511, 512, 1023] + sorted(rng.choice(np.arange(260, 1000), 34, replace=False).tolist())
    cnt, lens = np.zeros(n, int), np.zeros(n, int)
    cnt[at], lens[at] = rng.integers(1, 4, len(at)), rng.integers(4, 300, len(at))
    lens[512], lens[256] = 5000, 1700
    pool = Pool(380 + hd, 200, 1, hd, T)
    table = rng.integers(0, 200, (n, -(-5000 // T) + 1)).astype(np.int32)           # pages shared, as read-only ones may be
    R = int(cnt.sum()) + 2                                                           # the rows that run_attention passes
    assert bd_().bd_kv_attention_workspace(4, 1, hd, n, R, int(cnt.max()), T, table.shape[1]) > 0
    for ws in (True, False):
        got, ref, bound = run_attention(pool, lens, cnt, 1, 4, dtype, table=table, workspace=ws)
        assert (np.abs(got - ref) <= bound).all() and (got != 0).any(axis=(1, 2)).all()


@pytest.mark.parametrize("page", [32, 96])
def test_coded_decode_without_a_prompt(page):
    """No prompt at all: the window's own tokens are the cache's first, step by step against the float64 oracle with the same
    codes.  (Tolerances of one layer, derived in test_gpu_kv.py.)"""
    import tests.gpu_harness as gh
    from oracle.model import OracleModel
    bd = bd_()
    w, ws, prompts = small_model(n_layers=1)
    none = np.ascontiguousarray(prompts[:, :0])
    m = bd.Model(w, ws, DEV, kv="fp8", kv_page=page)
    tr = gh.capture_gpu_trace(m, none, w.gen_len, 0.9, 2, w.block_size, logits_for={0})
    rep = gh.lockstep(ok.with_coded_cache(OracleModel(w, ws, "f64"), page), none, [0], tr, w.gen_len, 0.9, 2, w.block_size, 5e-3, 3e-2)
    a, b = (bd.decode(m, none, w.gen_len, 0.9, 2, w.block_size) for _ in range(2))
    st = bd.State(m, none, w.gen_len, 0.9, 2, w.block_size)
    st.reset()                                                                       # (a prompt of no tokens ends at a page's end)
    st.close()
    m.close()
    assert all((x == y).all() for x, y in zip(a, b))
    assert not rep.failures and rep.complete, rep
