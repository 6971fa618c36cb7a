"""CPU checks of what the `kv` grid of the sweep goes by."""
from bd_synth import Workload


def workload(**kw):
    d = dict(n_layers=3, d_model=256, n_heads=4, n_kv_heads=4, head_dim=64, ffn_dim=512, vocab=1024, dtype="bf16", batch=5,
             prompt_len=40, block_size=4, n_inflight=1, gen_len=60)
    return Workload("ks", 1, **dict(d, **kw))


def test_cache_bytes_count_the_rows_that_no_buffer_holds():
    """K and V rows of a forward, fp32, where the FFN's rows are shorter than theirs."""
    from paper_2609_33887_amd.sweep import cache_bytes
    coded = 2 * 3 * 5 * 4 * 4 * (32 * 64 + 4)                                       # layers, sequences, kv heads, pages of 32
    assert cache_bytes(workload(), "fp8") == coded                                  # 512 a row in buffers of 512
    assert cache_bytes(workload(ffn_dim=384), "fp8") == coded + 256 * 512 * 4       # 5 * 40 rows, in 256s
    assert cache_bytes(workload(ffn_dim=384, block_size=20, n_inflight=3), "fp8") == coded + 768 * 512 * 4   # windows of 5 * 120
    moe = dict(n_experts=8, top_k=2, expert_ffn=128, n_shared=1, ffn_dim=0)
    assert cache_bytes(workload(**moe), "fp8") == coded
    assert cache_bytes(workload(**dict(moe, top_k=1)), "fp8") == coded + 256 * 512 * 4
    assert cache_bytes(workload(ffn_dim=384)) == cache_bytes(workload())


def test_precision_sweep_names_what_it_counts(monkeypatch):
    """Weight bytes only where the weights are what is compared; the least memory among the valid ones is deployed."""
    import numpy as np
    from paper_2609_33887_amd import sweep
    toks = np.arange(40 * 60).reshape(40, 60)
    monkeypatch.setattr(sweep, "decode_all", lambda model, prompts, G, cfg, B, batch: (toks, np.full(40, 12)))
    w = workload()
    run = lambda names, memory: sweep.precision_sweep(w, dict.fromkeys(names), None, 60, 4, (names[0], (0.9, 1)),
                                                      [(names[1], (0.9, 1))], 0.1, 0.1, memory=memory)
    r = run(("pair", "kv-fp8"), lambda p: sweep.cache_bytes(w, "fp8" if p == "kv-fp8" else None))
    assert "weight_bytes" not in r and r["memory_bytes"] == [sweep.cache_bytes(w), sweep.cache_bytes(w, "fp8")]
    assert r["selected"] == 1
    r = run(("bf16", "fp8"), None)
    assert r["weight_bytes"] == r["memory_bytes"] == [sweep.weight_bytes(w), sweep.weight_bytes(w, "fp8")]
