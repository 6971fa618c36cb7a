"""The paged attention's numbers against float64: outputs that are off by their own rounding alone, scales at both ends
of their range, and the query pairs that the models' decoding takes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import kv as ok
from tests.test_gpu_kv import DEV, U, Pool, attn_bound, bd_, dev, host, run_attention, starts

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def computed_bound(ref, mag, big, hd, keys):
    """attn_bound's error before the output's rounding, for bf16 calls as for fp32 ones: weights of two fp16 parts, 2^-21."""
    return attn_bound(ref, mag, big, hd, keys, torch.float32)


# lengths, rows, q-heads, kv-heads, head size, page, block, columns of the table behind the longest request (the kernel's
# form goes by the table and the rows): one query group of eight waves, whole and with its keys cut into ranges; two groups;
# four
FORMS = [([1057], [1], 16, 4, 128, 32, 1, 2), ([1057], [1], 16, 16, 64, 32, 1, 2), ([1440] * 3, [96] * 3, 16, 4, 128, 32, 32, 2),
         ([9000, 40], [1, 5], 16, 4, 128, 64, 1, 2), ([2500] * 2, [64] * 2, 16, 4, 128, 32, 64, 2),
         ([300] * 6, [96] * 6, 16, 16, 64, 32, 32, 2), ([1100, 640, 900, 400], [400, 640, 300, 77], 16, 8, 128, 64, 32, 2),
         ([2100] + [200] * 5, [96] * 6, 16, 16, 64, 32, 32, 2),
         ([700, 640, 700, 400], [700, 640, 700, 77], 16, 8, 128, 64, 32, 2), ([1500] + [130] * 5, [96] * 6, 16, 16, 64, 32, 32, 256),
         ([1500] + [130] * 5, [96] * 6, 16, 16, 128, 32, 32, 256)]


@pytest.mark.parametrize("i", range(len(FORMS)))
def test_bf16_outputs_are_the_rounded_float64_ones(i):
    """An output lies between the roundings of the float64 value less and plus what fp32 arithmetic is off by.

    Weights of 11 bits move one output in thirty to the next bfloat16 value, 8e-4 of the outputs' norm.  Scores in fp32
    (sums of hd terms: sqrt(hd) 2^-24 of a size of about 5, then 2^-22 of v_exp_f32) leave weights off by some 1e-6 and
    an output by 3e-6 at most, each key's error its own: 2 * 3e-6 of a step of 2^-8 is a share of 1.5e-3 moved by 2^-7 of
    themselves at most, sqrt(1.5e-3) 2^-7 = 3e-4 of the norm."""
    lens, cnt, H, Hkv, hd, T, B, spare = FORMS[i]
    pool = Pool(300 + i, sum(-(-x // T) for x in lens) + 2, Hkv, hd, T, spread=1)
    table = pool.tables(lens, spare)
    got, ref, _ = run_attention(pool, lens, cnt, B, H, torch.bfloat16, seed=i, table=table)
    q = np.random.default_rng([5, i]).standard_normal((sum(cnt), H, hd))
    q = host(dev(q, torch.float32).to(torch.bfloat16))
    again, mag, big = ok.attention(pool.kc, pool.ks, pool.vc, pool.vs, q, table, starts(cnt), np.array(lens) - cnt, lens, B)
    assert (again == ref).all()
    e = computed_bound(ref, mag, big, hd, max(lens))
    assert ((got >= bf16(ref - e)) & (got <= bf16(ref + e))).all(), float(np.mean((got < bf16(ref - e)) | (got > bf16(ref + e))))
    off = np.linalg.norm(got - bf16(ref)) / np.linalg.norm(ref)
    print(f"form {i}: {off:.2e} of the norm, {np.mean(got != bf16(ref)):.2e} of the outputs")
    assert off <= 3e-4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_small_weights_of_pages_of_far_larger_values(dtype):
    """Weights of 2^-105.5 times values of 2^10 beside weights of 1 times values of 2^-100: the first are 2^4.5 times the second,
    whatever reference the weights are held against."""
    hd, T = 64, 32
    pool = Pool(340, 10, 1, hd, T)
    pool.kc[:] = 0
    pool.ks[:] = 1.0
    pool.vs[:], pool.vs[9] = 2.0 ** -100, 2.0 ** 10
    # the other page's keys: scores of -72 * 8.125 / 8, -105.5 in log2 units (every number exact in its type)
    q0 = 8.125
    pool.kc[9, 0, :, 0] = ok.e4m3_code(-72.0)
    q = np.zeros((1, 2, hd))
    q[..., 0] = q0
    for order in ([0, 1, 2, 3, 4, 5, 6, 7, 9], [9, 1, 2, 3, 4, 5, 6, 7, 8]):        # a wave takes every eighth of the keys' tiles
        table = np.array([order], dtype=np.int32)
        qt = dev(q, torch.float32).to(dtype)
        o = bd_().kv_attention(pool.cache(), qt, dev(table), dev([0, 1]), dev([287]), dev([288]), 1)
        ref, mag, big = ok.attention(pool.kc, pool.ks, pool.vc, pool.vs, q, table, [0, 1], [287], [288], 1)
        assert (np.abs(host(o) - ref) <= attn_bound(ref, mag, big, hd, 288, dtype)).all(), order


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd,lens", [(64, [3]), (128, [70, 33]), (128, [5000])])
def test_values_of_the_smallest_scales(hd, lens, dtype):
    """Pages whose V scale is far below what an exponential of float32 reaches from the weights' reference (2^-126)."""
    pool = Pool(350 + hd + len(lens), sum(-(-x // 32) for x in lens) + 1, 2, hd, 32)
    for E in (-126, -120, -113, 119):
        pool.vs[:] = 2.0 ** E
        got, ref, bound = run_attention(pool, lens, [1] * len(lens), 1, 4, dtype, workspace=True)
        # below the type's normal numbers a rounding is half of its smallest one
        bound = bound + 0.5 * torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        assert (np.abs(got - ref) <= bound).all(), (E, np.max(np.abs(got - ref) / bound))
        assert (got != 0).any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ks,q0,scale", [(-126, 118, 0.0), (-100, 116, 2.0 ** -40), (28, -126, 2.0 ** 100), (-20, -80, 2.0 ** 100)])
def test_scores_where_scale_times_page_scale_leaves_float32(ks, q0, scale, dtype):
    """The product of the scores' factor and a page's K scale under 2^-126 or past 2^128, while the scores are ordinary ones; a
    query of zeros beside the others."""
    hd, T = 64, 32
    pool = Pool(360, 4, 1, hd, T)
    pool.ks[:] = 2.0 ** ks
    table = np.array([[2, 0, 3]], dtype=np.int32)
    q = np.zeros((2, 3, hd))
    q[:, 0, 0], q[:, 1, 0], q[:, 1, 5] = 2.0 ** q0, -2.0 ** q0, 2.0 ** q0
    pool.vc[2, 0, 4, 9] = 0x7F                                                      # a NaN that every query sees
    o = bd_().kv_attention(pool.cache(), dev(q, torch.float32).to(dtype), dev(table), dev([0, 2]), dev([75]), dev([77]), 1, scale=scale)
    ref, mag, big = ok.attention(pool.kc, pool.ks, pool.vc, pool.vs, q, table, [0, 2], [75], [77], 1, scale=scale or None)
    bound = attn_bound(ref, mag, big, hd, 77, dtype)
    bad = np.isnan(ref)
    assert bad.sum() == 6 and (np.isnan(host(o)) == bad).all()
    assert (np.abs(host(o) - ref)[~bad] <= bound[~bad]).all(), np.nanmax(np.abs(host(o) - ref) / bound)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pages_beside_one_whose_factor_leaves_float32(dtype):
    """One page at the lowest scale among ordinary ones (two tiles a stage in the form that many rows take), and a scale
    argument so large that the ordinary pages' scores would leave float32 without their own scale."""
    hd, T, n = 64, 32, 40
    pool = Pool(365, 4, 16, hd, T)
    pool.kc[:] = ok.e4m3_code(np.abs(pool.rng.standard_normal(pool.kc.shape)) * 60.0 + 1)
    table = np.tile(np.array([[2, 0, 3]], dtype=np.int32), (n, 1))
    q = np.zeros((100 * n, 16, hd))
    q[..., 3] = 1.0
    for scale, ks in ((0.0, (-3, -126, -3)), (2.0 ** 126, (-125, 10, -124))):
        for p, e in zip(table[0], ks):
            pool.ks[p] = 2.0 ** e
        if scale:
            pool.kc[0] = 0                                                          # its scores are 0, whatever its scale
        qt = dev(q, torch.float32).to(dtype)
        start = np.arange(n + 1) * 100
        o = bd_().kv_attention(pool.cache(), qt, dev(table), dev(start), dev(np.zeros(n)), dev(np.full(n, 77)), 0, scale=scale, max_rows=100)
        few = slice(0, 100)
        ref, mag, big = ok.attention(pool.kc, pool.ks, pool.vc, pool.vs, q[few], table[:1], [0, 100], [0], [77], 0, scale=scale or None)
        bound = attn_bound(ref, mag, big, hd, 77, dtype)
        assert (np.abs(host(o[few]) - ref) <= bound).all(), np.max(np.abs(host(o[few]) - ref) / bound)
        assert torch.equal(o.view(n, 100, 16, hd), o[:100].expand(n, 100, 16, hd))
