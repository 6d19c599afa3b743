"""The KV cache in 8 bits, without a GPU: pins of its oracle, refusals of its calls, argument types."""
import numpy as np
import pytest

import paper_2412_12488_amd as mc
from oracle import kv8

FAKE = 0x10000                 # a non-null, aligned "device address" that is never dereferenced


def test_numbers_are_the_formats():
    import torch
    ref = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(kv8.NUMBERS, ref, equal_nan=True)


def test_rounding_is_to_the_nearest_and_even():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-12, 8, 4000), kv8.POSITIVE,
                        (kv8.POSITIVE[1:] + kv8.POSITIVE[:-1]) / 2, [0.0, -0.0, 448.0, 2.0 ** -11]])
    x = np.clip(np.concatenate([x, -x]), -448, 448)
    codes = kv8.round_codes(x)
    got = kv8.NUMBERS[codes]
    away = np.abs(kv8.POSITIVE[None] - np.abs(x)[:, None])
    best = away.min(1)
    assert np.array_equal(np.abs(np.abs(got) - np.abs(x)), best)
    ties = (away == best[:, None]).sum(1) > 1
    assert ties.sum() > 200 and np.all(codes[ties] % 2 == 0)
    assert kv8.round_codes(np.array([np.nan]))[0] == 0x7f


@pytest.mark.parametrize("dtype", [kv8.F16, kv8.BF16])
def test_scale_is_the_least_that_holds_the_block_and_values_fit_the_type(dtype):
    import torch
    lo, hi = kv8.LIMITS[dtype]
    for big in (0.0, 1e-30, 2.0 ** -24, 0.01, 0.875, 1.0, 1.75, 1.7500001, 3.9, 448.0, 448.5, 57344.0, 60000.0, 65504.0):
        k = kv8.scale_exponent(np.array([big, -big / 2]), dtype)
        assert lo <= k <= hi
        assert big <= 448 * 2.0 ** k or k == hi
        assert k == lo or big > 448 * 2.0 ** (k - 1)
    # every code at every scale is a number of the 16-bit type
    t = torch.float16 if dtype == kv8.F16 else torch.bfloat16
    for k in (lo, lo + 1, 0, hi - 1, hi):
        v = kv8.NUMBERS[~np.isnan(kv8.NUMBERS)] * 2.0 ** k
        if k == hi:
            v = v[np.abs(v) <= 240 * 2.0 ** k]
        v = torch.from_numpy(v)
        assert torch.equal(v.to(t).double(), v)
    big = float(torch.finfo(t).max)
    assert kv8.NUMBERS[kv8.encode(np.array([big]), hi, dtype)][0] == 240


def test_append_token_by_token_is_within_a_rounding_of_at_once():
    """Codes that move to a larger scale are rounded twice: at most once and a half half-steps off."""
    rng = np.random.default_rng(1)
    bits = (rng.normal(size=(40, 1, 128)) * 2.0 ** rng.integers(-6, 6, (40, 1, 1))).astype(np.float16).view(np.uint16)
    one, all_ = kv8.Pool(1, 4, 1, kv8.F16), kv8.Pool(1, 4, 1, kv8.F16)
    for i in range(40):
        one.append(0, bits[i:i + 1], bits[i:i + 1], 5 + i, [3, 1, 2])
    all_.append(0, bits, bits, 5, [3, 1, 2])
    assert np.array_equal(one.k[:, 1:4], all_.k[:, 1:4])
    a, b = one.values(0, [3, 1, 2], 45)[0][0][5:], all_.values(0, [3, 1, 2], 45)[0][0][5:]
    step = 2.0 ** -3 * np.abs(b) + 2.0 ** -9 * 2.0 ** all_.k.max()
    assert np.all(np.abs(a - b) <= step)


def test_attention_oracle_against_two_keys_by_hand():
    pool = kv8.Pool(1, 2, 1, kv8.BF16)
    k = np.zeros((2, 1, 128), np.uint16)
    v = np.zeros((2, 1, 128), np.uint16)
    k[1, 0, 0], v[0, 0, 3], v[1, 0, 3] = 0x3f80, 0x3f80, 0x4000        # 1; 1, 2
    pool.append(0, k, v, 0, [1])
    q = np.zeros((2, 1, 128), np.uint16)
    q[:, 0, 0] = 0x4000                                                 # 2
    out, lse, *_ = kv8.attention(pool, 0, [1], q, 0, scale=0.5)
    e = np.e
    assert np.allclose(out[:, 0, 3], [1.0, (1 + 2 * e) / (1 + e)], rtol=1e-14)
    assert np.allclose(lse[:, 0], [0.0, np.log(1 + e)], rtol=1e-14, atol=1e-16)


# ---- refusals ----
def pool8(**kw):
    d = dict(codes=FAKE, scales=FAKE, num_layers=2, num_pages=8, num_kv_heads=2, dtype=mc.MC_BF16)
    d.update(kw)
    return mc.pool8_desc(**d)


def pool16(**kw):
    d = dict(base=FAKE, num_layers=2, num_pages=8, num_kv_heads=2, dtype=mc.MC_BF16)
    d.update(kw)
    return mc.pool_desc(**d)


def status(fn, *args):
    try:
        fn(*args, 0)
        return mc.MC_OK
    except mc.McError as e:
        return e.status


BAD_POOLS = [(dict(codes=0), mc.MC_ERR_INVALID), (dict(scales=0), mc.MC_ERR_INVALID),
             (dict(codes=FAKE + 8), mc.MC_ERR_INVALID), (dict(scales=FAKE + 4), mc.MC_ERR_INVALID),
             (dict(skipped=FAKE + 2), mc.MC_ERR_INVALID), (dict(num_layers=0), mc.MC_ERR_INVALID),
             (dict(num_pages=-1), mc.MC_ERR_INVALID), (dict(num_kv_heads=0), mc.MC_ERR_INVALID),
             (dict(page_size=32), mc.MC_ERR_UNSUPPORTED), (dict(head_dim=64), mc.MC_ERR_UNSUPPORTED),
             (dict(dtype=2), mc.MC_ERR_UNSUPPORTED)]


@pytest.mark.parametrize("bad, want", BAD_POOLS)
def test_every_call_refuses_a_bad_pool(bad, want):
    p = pool8(**bad)
    ws = mc.mc_attn8_workspace_size(1, 1, 8, 2)
    assert status(mc.mc_kv8_append, p, 0, FAKE, FAKE, 1, 1, FAKE, FAKE, FAKE, FAKE) == want
    assert status(mc.mc_attn8_plan, p, 8, 1, 1, FAKE, FAKE, FAKE, FAKE, FAKE, ws) == want
    assert status(mc.mc_kv8_compress_range, pool16(), p, 0, 1, FAKE, 1, FAKE, 1, 0, 16) == want
    assert status(mc.mc_kv8_restore_range, p, pool16(), 0, 1, FAKE, 1, FAKE, 1, 0, 16) == want
    assert status(mc.mc_kv8_pack_range, p, 0, 1, FAKE, 1, 0, 16, FAKE) == want
    assert status(mc.mc_kv8_unpack_range, p, 0, 1, FAKE, 1, 0, 16, FAKE) == want
    assert status(mc.mc_kv8_copy_page, p, 0, 1, 0, 1) == want


def test_append_refusals():
    ok = [pool8(), 0, FAKE, FAKE, 1, 1, FAKE, FAKE, FAKE, FAKE]

    def call(**at):
        a = list(ok)
        for i, v in at.items():
            a[int(i[1:])] = v
        return status(mc.mc_kv8_append, *a)
    assert call(_1=2) == call(_1=-1) == mc.MC_ERR_RANGE
    assert call(_4=-1) == call(_5=-1) == mc.MC_ERR_INVALID
    for i in (2, 3, 6, 7, 8, 9):
        assert call(**{f"_{i}": 0}) == mc.MC_ERR_INVALID
    assert call(_2=FAKE + 8) == call(_3=FAKE + 8) == mc.MC_ERR_INVALID
    assert call(_4=0) == call(_5=0) == mc.MC_OK                       # nothing to do, nothing launched


def test_attention_refusals():
    size = mc.mc_attn8_workspace_size(2, 40, 8, 2)
    assert size > 0 and size % 16 == 0
    for bad in ((-1, 1, 8, 2), (1, -1, 8, 2), (1, 1, 0, 2), (1, 1, 8, 0), (1, 1, 7, 2), (1, 1, 6, 2), (1, 1, 32, 2)):
        assert mc.mc_attn8_workspace_size(*bad) == 0
    plan = [pool8(), 8, 2, 40, FAKE, FAKE, FAKE, FAKE, 0, FAKE, size]

    def planned(**at):
        a = list(plan)
        for i, v in at.items():
            a[int(i[1:])] = v
        return status(mc.mc_attn8_plan_ahead, *a)
    assert planned(_1=6) == planned(_1=7) == planned(_1=32) == mc.MC_ERR_UNSUPPORTED
    assert planned(_1=0) == planned(_2=-1) == planned(_3=-1) == mc.MC_ERR_INVALID
    assert planned(_8=-1) == planned(_8=(1 << 20) + 1) == mc.MC_ERR_RANGE
    assert planned(_9=0) == planned(_9=FAKE + 4) == planned(_10=size - 1) == mc.MC_ERR_INVALID
    for i in (4, 5, 6, 7):
        assert planned(**{f"_{i}": 0}) == mc.MC_ERR_INVALID
    attn = [pool8(), 0, FAKE, 8, 2, 40, FAKE, FAKE, FAKE, FAKE, 0.0, FAKE, FAKE, FAKE, size]

    def attend(**at):
        a = list(attn)
        for i, v in at.items():
            a[int(i[1:])] = v
        return status(mc.mc_prefix_prefill_attn8, *a)
    assert attend(_1=2) == attend(_1=-1) == mc.MC_ERR_RANGE
    assert attend(_3=6) == mc.MC_ERR_UNSUPPORTED
    for bad in (-1.0, float("nan"), float("inf")):
        assert attend(_10=bad) == mc.MC_ERR_INVALID
    for i in (2, 6, 7, 8, 9, 11, 12, 13):
        assert attend(**{f"_{i}": 0}) == mc.MC_ERR_INVALID
    assert attend(_2=FAKE + 8) == attend(_11=FAKE + 8) == attend(_12=FAKE + 2) == attend(_13=FAKE + 8) == mc.MC_ERR_INVALID
    assert attend(_14=size - 1) == mc.MC_ERR_INVALID
    assert attend(_4=0) == attend(_5=0) == mc.MC_OK
    assert mc.lib().mc_attn8_plan_check(None, None) == mc.MC_ERR_INVALID


@pytest.mark.parametrize("name", ["compress", "restore"])
def test_conversion_refusals(name):
    fn = getattr(mc, f"mc_kv8_{name}_range")
    a, b = (pool16, pool8) if name == "compress" else (pool8, pool16)

    def call(l0=0, l1=2, t0=FAKE, n0=4, t1=FAKE, n1=4, s0=16, s1=50, p=None, r=None):
        return status(fn, p or a(), r or b(), l0, l1, t0, n0, t1, n1, s0, s1)
    assert call(l0=-1) == call(l0=2, l1=1) == call(l1=3) == mc.MC_ERR_RANGE
    assert call(s0=-16) == call(s0=64, s1=50) == call(n0=-1) == call(n1=-1) == mc.MC_ERR_RANGE
    assert call(n0=3) == call(n1=3) == mc.MC_ERR_RANGE                 # a table does not cover token s1 - 1
    assert call(t0=0) == call(t1=0) == mc.MC_ERR_INVALID
    assert call(s0=48, s1=48) == call(l0=1, l1=1) == mc.MC_OK
    if name == "compress":
        assert call(s0=17) == mc.MC_ERR_RANGE
    assert call(p=a(dtype=mc.MC_F16)) == call(p=a(num_kv_heads=4)) == mc.MC_ERR_UNSUPPORTED
    assert call(r=b(num_layers=1)) == call(p=a(num_layers=1)) == mc.MC_ERR_RANGE


@pytest.mark.parametrize("name", ["pack", "unpack"])
def test_transfer_refusals(name):
    fn = getattr(mc, f"mc_kv8_{name}_range")

    def call(l0=0, l1=2, t=FAKE, n=4, s0=16, s1=50, buf=FAKE):
        return status(fn, pool8(), l0, l1, t, n, s0, s1, buf)
    assert call(l0=-1) == call(l0=2, l1=1) == call(l1=3) == mc.MC_ERR_RANGE
    assert call(s0=-16) == call(s0=64, s1=50) == call(n=-1) == call(n=3) == call(s0=17) == mc.MC_ERR_RANGE
    assert call(t=0) == call(buf=0) == call(buf=FAKE + 8) == mc.MC_ERR_INVALID
    assert call(s0=48, s1=48) == call(l0=1, l1=1) == mc.MC_OK


def test_page_copy_refusals():
    def call(l0=0, l1=2, src=0, dst=1):
        return status(mc.mc_kv8_copy_page, pool8(), l0, l1, src, dst)
    assert call(l0=-1) == call(l1=3) == call(src=8) == call(dst=-1) == mc.MC_ERR_RANGE
    assert call(dst=0) == mc.MC_ERR_ALIAS
    assert call(l0=1, l1=1) == mc.MC_OK
    assert mc.lib().mc_kv8_copy_check(None, None, None) == mc.MC_ERR_INVALID


def test_descriptors_of_the_two_pools_are_not_taken_for_each_other():
    with pytest.raises(mc.binding.McArgumentError):
        mc.mc_kv8_append(pool16(), 0, FAKE, FAKE, 1, 1, FAKE, FAKE, FAKE, FAKE, 0)
    with pytest.raises(mc.binding.McArgumentError):
        mc.mc_kv_append(pool8(), 0, FAKE, FAKE, 1, 1, FAKE, FAKE, FAKE, FAKE, 0)
    with pytest.raises(mc.binding.McArgumentError):
        mc.mc_kv8_restore_range(pool16(), pool8(), 0, 1, FAKE, 1, FAKE, 1, 0, 16, 0)
