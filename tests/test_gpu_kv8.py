"""The KV cache in 8 bits on the GPU, against the oracle in 64 bits (oracle/kv8.py).

Codes and scales are compared for equality.  Attention: with u = half the 16-bit type's epsilon (what a rounding
to nearest loses), P is rounded once (u A, A = sum_j p_j |v_j|) and the result once (u |out|); a score is a sum of 128
products in fp32, off by at most 130 x 2^-24 E (E: the largest sum of |products|), which moves p_j and the sum by that much
relative, and exp2 and its argument by a few 2^-24 of the argument, whose size is at most E + |lse|; fp16 holds
small p in steps of 2^-24, half of which for each key of the row costs 2^-25 V.  The factors are rounded up to twice."""
import numpy as np
import pytest

import paper_2412_12488_amd as mc
from oracle import kv8

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {kv8.F16: torch.float16, kv8.BF16: torch.bfloat16}
BOTH = pytest.mark.parametrize("dtype", [kv8.BF16, kv8.F16], ids=["bf16", "fp16"])


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).to(DEV)


def cu(lens):
    return dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))


def normal_bits(rng, shape, dtype, spread=0):
    x = rng.normal(size=shape)
    if spread:
        x = x * 2.0 ** rng.integers(-spread, spread + 1, shape[:1] + (1,) * (len(shape) - 1))
    return torch.from_numpy(x).to(TYPES[dtype]).view(torch.int16).numpy().view(np.uint16)


class Case:
    """Pages dealt at random, an 8-bit pool whose every byte is `fill` (NaN codes, unless said otherwise) on the GPU,
    and the oracle's pool of the same bytes."""

    def __init__(self, rng, dtype, heads, begin, new, layers=1, spare=3, fill=0x7f, tables=None):
        self.rng, self.dtype, self.heads, self.layers = rng, dtype, heads, layers
        self.begin, self.new = np.array(begin), np.array(new)
        need = -(-(self.begin + self.new) // 16)
        self.num_pages = int(need.sum()) + spare
        ids = rng.permutation(self.num_pages).astype(np.int32)
        cut = np.concatenate([[0], np.cumsum(need)])
        self.tables = tables or [ids[cut[i]:cut[i + 1]] for i in range(len(need))]
        raw = np.full((layers, self.num_pages, 2, heads, 2048), fill, np.uint8)
        scales = np.full((layers, self.num_pages, heads, 2), 1.0, np.float32)
        self.o = kv8.Pool(layers, self.num_pages, heads, dtype, raw, scales)
        self.upload()

    def upload(self):
        raw, scales = self.o.raw()
        self.codes, self.scales = dev(raw), dev(scales)
        self.skipped = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.desc = mc.pool8_desc(self.codes, self.scales, self.layers, self.num_pages, self.heads, self.dtype,
                                  skipped=self.skipped)

    def batch(self, begin=None, new=None):
        begin, new = self.begin if begin is None else np.array(begin), self.new if new is None else np.array(new)
        self.args = [len(new), int(new.sum()), cu(new), dev(begin.astype(np.int32)),
                     dev(np.concatenate(self.tables).astype(np.int32)), cu([len(t) for t in self.tables])]
        return self.args

    def fill(self, layer=0, upto=None, spread=0):
        """The cached tokens of every sequence, through the oracle, then up."""
        for s, b in enumerate(self.begin if upto is None else upto):
            if b:
                k, v = (normal_bits(self.rng, (int(b), self.heads, 128), self.dtype, spread) for _ in range(2))
                self.o.append(layer, k, v, 0, self.tables[s])
        self.upload()

    def new_kv(self, spread=0):
        return [normal_bits(self.rng, (int(self.new.sum()), self.heads, 128), self.dtype, spread) for _ in range(2)]

    def oracle_append(self, k, v, layer=0):
        at = 0
        for s, n in enumerate(self.new):
            if n:
                self.o.append(layer, k[at:at + n], v[at:at + n], int(self.begin[s]), self.tables[s])
            at += n

    def same(self):
        """Codes (a NaN is a NaN) and scales of the whole pool."""
        raw, scales = self.o.raw()
        got = self.codes.cpu().numpy()
        nan = np.isnan(kv8.NUMBERS)
        bad = (got != raw) & ~(nan[got] & nan[raw])
        assert not bad.any(), f"{bad.sum()} codes differ, first at {np.argwhere(bad)[0]}"
        assert np.array_equal(self.scales.cpu().numpy(), scales)


def attend(c, q, hq, layer=0, scale=0.0, plan=mc.mc_attn8_plan, check=True):
    """out, lse of the batch that c.batch() made, rows that nothing writes NaN."""
    B, tq = c.args[:2]
    size = mc.mc_attn8_workspace_size(B, tq, hq, c.heads)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((tq, hq, 128), float("nan"), dtype=TYPES[c.dtype], device=DEV)
    lse = torch.full((tq, hq), float("nan"), device=DEV)
    plan(c.desc, hq, *c.args, ws, size)
    if check:
        mc.mc_attn8_plan_check(ws)
    for _ in range(2):                     # the second run finds what the first left in the workspace
        mc.mc_prefix_prefill_attn8(c.desc, layer, q, hq, *c.args, scale, out, lse, ws, size)
    torch.cuda.synchronize()
    return out, lse, ws


def close(got, got_lse, want, dtype, n_keys):
    out, lse, A, E, V = want
    u = 2.0 ** (-8 if dtype == kv8.BF16 else -11)
    small = 2 * (130 * 2.0 ** -24 * E + 8 * 2.0 ** -24 * (E + np.abs(lse) + 1) + n_keys * 2.0 ** -24)
    tol = (1.01 * u + 2 * small)[..., None] * A + 1.01 * u * np.abs(out) + 2.0 ** -24
    if dtype == kv8.F16:
        tol = tol + (n_keys * 2.0 ** -25 * V)[..., None]
    else:
        tol = tol + 0
    err = np.abs(got - out)
    assert np.all(err <= tol), f"out: off by {np.nanmax(err)}, {np.nanmax(err / tol)} of the tolerance, at {np.unravel_index(np.nanargmax(err / tol), err.shape)}"
    err = np.abs(got_lse - lse)
    assert np.all(err <= small + 2.0 ** -20), f"lse: off by {np.nanmax(err)}"


def check_attention(c, q, hq, out, lse, layer=0, scale=None, sample=24):
    """Rows of every sequence (all, or some with the first and the last) against the oracle."""
    at = 0
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for s, n in enumerate(c.args_new):
        if n:
            rows = np.arange(n) if n <= sample else np.unique(np.concatenate(
                [[0, 1, n - 2, n - 1], c.rng.integers(0, n, sample)]))
            want = kv8.attention(c.o, layer, c.tables[s], q[at:at + n], int(c.args_begin[s]), scale, rows)
            close(got[at + rows], got_lse[at + rows], want, c.dtype, int(c.args_begin[s]) + n)
        at += n


def run_attention(c, hq, scale=None, q_gain=1.0, sample=24, **kw):
    c.args_begin, c.args_new = c.begin, c.new
    c.batch()
    q = normal_bits(c.rng, (int(c.new.sum()), hq, 128), c.dtype)
    out, lse, _ = attend(c, dev(q).view(TYPES[c.dtype]), hq, scale=0.0 if scale is None else scale, **kw)
    check_attention(c, q, hq, out, lse, scale=scale, sample=sample)
    return q, out, lse


# ---------------------------------------------------------------- append -----
@BOTH
@pytest.mark.parametrize("shuffled", [False, True])
def test_every_16_bit_pattern(dtype, shuffled):
    """All 65536 numbers, infinities and NaNs among them, in pages of like and of mixed magnitudes."""
    rng = np.random.default_rng(1)
    bits = np.arange(65536, dtype=np.uint16)
    if shuffled:
        rng.shuffle(bits)
    c = Case(rng, dtype, 1, [0], [512])
    k, v = bits.reshape(512, 1, 128), bits[::-1].copy().reshape(512, 1, 128)
    mc.mc_kv8_append(c.desc, 0, dev(k), dev(v), *c.batch())
    c.oracle_append(k, v)
    c.same()


@BOTH
@pytest.mark.parametrize("heads, begin, new", [
    (1, [0], [1]), (2, [15], [1]), (3, [16], [1]), (8, [7, 0, 33], [1, 1, 1]), (5, [3, 31, 0], [9, 0, 17]),
    (8, [100, 0, 5, 48], [40, 16, 300, 1]), (2, [13, 250], [900, 700]), (4, list(range(70)), [1] * 70),
    (1, [0, 9], [1600, 1]), (2, [5] * 300, [4] * 300)])
def test_append(dtype, heads, begin, new):
    rng = np.random.default_rng(2)
    c = Case(rng, dtype, heads, begin, new, layers=2)
    c.fill(layer=1, spread=4)
    k, v = c.new_kv(spread=4)
    mc.mc_kv8_append(c.desc, 1, dev(k), dev(v), *c.batch())
    c.oracle_append(k, v, layer=1)
    c.same()
    assert c.skipped.item() == 0


@pytest.mark.parametrize("heads, begin, new", [
    (24, [3, 0], [1100, 400]), (24, [7] * 200 + [40], [1] * 200 + [1300]), (3, [9] * 90 + [5], [1, 0, 0] * 30 + [170]),
    (24, [5, 0, 30] * 40 + [0], [3, 0, 1] * 40 + [1500])])
def test_append_by_workgroups_of_many_tokens(heads, begin, new):
    test_append(kv8.BF16, heads, begin, new)


@BOTH
def test_append_token_by_token(dtype):
    """Scales that grow again and again, the old codes moved each time, to a factor that leaves nothing of them."""
    rng = np.random.default_rng(3)
    c = Case(rng, dtype, 2, [5], [40])
    c.fill()
    gain = 2.0 ** np.concatenate([rng.integers(-10, 4, 30), [-14, -12, 15, 15, -3, 0, 2, 4, 6, 8]])
    k = torch.from_numpy(rng.normal(size=(40, 2, 128)).clip(-1.9, 1.9) * gain[:, None, None]).to(TYPES[dtype])
    k = k.view(torch.int16).numpy().view(np.uint16)
    v = k[::-1].copy()
    for i in range(40):
        c.batch([5 + i], [1])
        mc.mc_kv8_append(c.desc, 0, dev(k[i]), dev(v[i]), *c.args)
        c.o.append(0, k[i:i + 1], v[i:i + 1], 5 + i, c.tables[0])
        if i % 7 == 0 or i > 30:
            c.same()
    c.same()


@pytest.mark.parametrize("new", [[3, 40, 5, 2], [700, 400, 300, 2]])
def test_append_leaves_out_what_has_no_place(new):
    """A page id outside the pool, a table that is too short, a negative begin; the others land."""
    rng = np.random.default_rng(4)
    c = Case(rng, kv8.BF16, 2, [20, 0, 4, 1], new)
    c.fill()
    k, v = c.new_kv()
    bad = [t.copy() for t in c.tables]
    bad[0][1] = c.num_pages
    c.batch()
    c.args[3] = dev(np.array([20, 0, -4, 1], np.int32))
    bad[1] = bad[1][:-1]
    c.args[4], c.args[5] = dev(np.concatenate(bad)), cu([len(t) for t in bad])
    mc.mc_kv8_append(c.desc, 0, dev(k), dev(v), *c.args)
    lost = min(new[0], 12) + (new[1] - 16 * len(bad[1])) + new[2]
    at = np.concatenate([[0], np.cumsum(new)])
    x = lambda i, lo, hi: (k[at[i] + lo:at[i] + hi], v[at[i] + lo:at[i] + hi])  # noqa: E731
    if new[0] > 12:
        c.o.append(0, *x(0, 12, new[0]), 32, c.tables[0])
    c.o.append(0, *x(1, 0, 16 * len(bad[1])), 0, c.tables[1])
    c.o.append(0, *x(3, 0, new[3]), 1, c.tables[3])
    c.same()
    assert mc.mc_kv8_copy_check(c.desc) == (mc.MC_ERR_RANGE, lost)
    assert mc.mc_kv8_copy_check(c.desc) == (mc.MC_OK, 0)


# -------------------------------------------------------------- attention ----
HEADS = [(8, 8), (4, 2), (8, 2), (8, 1)]       # groups of 1, 2, 4, 8


@BOTH
@pytest.mark.parametrize("hq, hkv", HEADS)
@pytest.mark.parametrize("begin, new", [
    ([0], [1]), ([63], [1]), ([64, 0, 200], [1, 1, 1]), ([1000], [1]), ([0], [2]), ([62], [3]),
    ([40, 500], [16, 17]), ([0, 7], [33, 129]), ([15, 0, 0, 300], [5, 0, 1, 64])])
def test_attention_small(dtype, hq, hkv, begin, new):
    rng = np.random.default_rng(5)
    c = Case(rng, dtype, hkv, begin, new)
    c.fill(upto=c.begin + c.new, spread=1)
    run_attention(c, hq)


@BOTH
@pytest.mark.parametrize("hq, hkv", HEADS)
@pytest.mark.parametrize("begin, new", [
    ([40, 500, 0, 15, 9, 300, 63], [16, 17, 5, 270, 0, 1, 2]), ([0, 62, 7], [33, 3, 229]), ([130], [64]), ([700], [65])])
def test_attention_of_short_and_long_ranges(dtype, hq, hkv, begin, new):
    """Q tiles of 16 and of 128 rows in one batch; batches at the border between the two kinds of plan."""
    test_attention_small(dtype, hq, hkv, begin, new)


@BOTH
@pytest.mark.parametrize("hq, hkv, begin, new", [
    (8, 2, [9000], [1]), (8, 1, [5000], [7]), (4, 4, [3000, 10, 999], [1, 1, 1]),
    (8, 2, list(range(0, 2600, 13)), [1] * 200), (16, 2, [2000], [130]), (8, 2, [1500], [500]),
    (4, 4, [0, 100], [700, 40]), (8, 8, [0, 512, 3, 77], [200, 1, 350, 1]), (8, 1, [600] * 5, [2, 1, 1, 40, 3]),
    (2, 1, [0], [2500])])
def test_attention(dtype, hq, hkv, begin, new):
    """Long contexts and batches: q tiles in several parts, parts of several q tiles in one span."""
    rng = np.random.default_rng(6)
    c = Case(rng, dtype, hkv, begin, new)
    c.fill(upto=c.begin + c.new, spread=1)
    run_attention(c, hq, sample=6)


@BOTH
@pytest.mark.parametrize("scale, spread", [(1.0, 0), (0.01, 0), (None, 3), (12.0, 0)])
def test_attention_of_other_scales(dtype, scale, spread):
    """Scores of a standard deviation of 11 (rows whose maximum moves far), of 0.1, of keys of many sizes, and of 140 (rows
    whose later keys beat the first ones by more than 2^60 in the exponent)."""
    rng = np.random.default_rng(7)
    c = Case(rng, dtype, 2, [700, 20, 1100], [3, 150, 40])
    c.fill(upto=c.begin + c.new, spread=spread)
    run_attention(c, 8, scale=scale)


@BOTH
@pytest.mark.parametrize("new", [1, 90])
def test_queries_of_many_sizes(dtype, new):
    """Numbers of a row of q from 2^-12 to 2^12 of each other, d by d, each d with keys of the other size; rows of zeros."""
    rng = np.random.default_rng(23)
    c = Case(rng, dtype, 2, [333], [new])
    n = 333 + new
    by = 2.0 ** rng.integers(-6, 7, 128)
    k = torch.from_numpy(rng.normal(size=(n, 2, 128)) / by).to(TYPES[dtype]).view(torch.int16).numpy().view(np.uint16)
    c.o.append(0, k, normal_bits(rng, (n, 2, 128), dtype), 0, c.tables[0])
    c.upload()
    c.args_begin, c.args_new = c.begin, c.new
    c.batch()
    x = rng.normal(size=(new, 8, 128)) * by
    x[new // 2, 3] = 0.0
    q = torch.from_numpy(x).to(TYPES[dtype]).view(torch.int16).numpy().view(np.uint16)
    out, lse, _ = attend(c, dev(q).view(TYPES[dtype]), 8)
    check_attention(c, q, 8, out, lse)


@pytest.mark.parametrize("new", [[1, 4], [100, 40]])
@pytest.mark.parametrize("code", [0x7f, 0xff, 0x7e])
def test_nothing_hidden_counts(new, code):
    """What keys a row must not see hold - NaN, the largest numbers - changes no bit of it: slots behind the
    last token and, for earlier rows, K and V of later tokens.  Rows that see a NaN in V have it in that d alone."""
    rng = np.random.default_rng(8)
    c = Case(rng, kv8.BF16, 2, [70, 301], new, fill=0)
    c.fill(upto=c.begin + c.new)
    q, out, lse = run_attention(c, 8)
    s, n = 1, int(c.begin[1] + new[1])                      # sequence 1: the last token's K and V of head 0, and behind it
    page, slot = c.tables[s][(n - 1) // 16], (n - 1) % 16
    c.o.codes[0, page, :, :, slot + 1:] = code
    c.upload()
    c.batch()
    again, lse2, _ = attend(c, dev(q).view(torch.bfloat16), 8)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    if code == 0x7e:
        return
    c.o.codes[0, page, 1, 0, slot, 5] = code
    c.upload()
    again, lse2, _ = attend(c, dev(q).view(torch.bfloat16), 8)
    want = out.clone()
    want[-1, 0:4, 5] = float("nan")
    assert torch.equal(torch.isnan(again), torch.isnan(want))
    assert torch.equal(again.nan_to_num(7), want.nan_to_num(7)) and torch.equal(lse, lse2)
    c.o.codes[0, page, 0, 1, slot, 9] = code                # and a key: the row that sees it is lost, with its lse
    c.upload()
    again, lse2, _ = attend(c, dev(q).view(torch.bfloat16), 8)
    want[-1, 4:8] = float("nan")
    assert torch.equal(torch.isnan(again), torch.isnan(want))
    assert torch.isnan(lse2[-1, 4:8]).all() and torch.equal(lse2[:-1], lse[:-1]) and torch.equal(lse2[-1, :4], lse[-1, :4])


def test_shared_pages_and_another_layer():
    """Two sequences on one prefix's pages, in layer 2 of 3."""
    rng = np.random.default_rng(9)
    ids = rng.permutation(80).astype(np.int32)
    tables = [ids[:40], np.concatenate([ids[:32], ids[40:50]])]
    c = Case(rng, kv8.F16, 2, [630, 512], [10, 160], layers=3, spare=0, tables=tables)
    c.num_pages = 82
    c.o = kv8.Pool(3, 82, 2, kv8.F16)
    for s, n in ((0, 640), (1, 672)):
        k, v = (normal_bits(rng, (n, 2, 128), kv8.F16) for _ in range(2))
        at = 0 if s == 0 else 512
        c.o.append(2, k[at:], v[at:], at, tables[s])
    c.upload()
    c.args_begin, c.args_new = c.begin, c.new
    c.batch()
    q = normal_bits(rng, (170, 4, 128), kv8.F16)
    out, lse, _ = attend(c, dev(q).view(torch.float16), 4, layer=2)
    check_attention(c, q, 4, out, lse, layer=2)


def test_malformed_sequences_are_left_out_alone():
    rng = np.random.default_rng(10)
    c = Case(rng, kv8.BF16, 2, [40, 100, 7, 300], [1, 30, 2, 5])
    c.fill(upto=c.begin + c.new)
    c.args_begin, c.args_new = c.begin, c.new
    good = [t.copy() for t in c.tables]
    q = normal_bits(rng, (38, 8, 128), kv8.BF16)
    bad = [t.copy() for t in good]
    bad[1][2] = -1
    bad[3] = bad[3][:-1]
    c.batch()
    c.args[4], c.args[5] = dev(np.concatenate(bad)), cu([len(t) for t in bad])
    out, lse, ws = attend(c, dev(q).view(torch.bfloat16), 8, check=False)
    with pytest.raises(mc.McError) as e:
        mc.mc_attn8_plan_check(ws)
    assert e.value.status == mc.MC_ERR_RANGE
    lost = np.zeros(38, bool)
    lost[1:31] = lost[33:] = True
    assert torch.isnan(out[lost]).all() and torch.isnan(lse[lost]).all()
    c.batch()
    whole, whole_lse, _ = attend(c, dev(q).view(torch.bfloat16), 8)
    check_attention(c, q, 8, whole, whole_lse)
    c.args_new = np.array([1, 0, 2, 0])
    check_attention(c, q[~lost], 8, out[~lost], lse[~lost])


@BOTH
def test_decode_batches_with_a_few_longer_ranges(dtype):
    """No more new tokens than sequences, but some have several q tiles of 16 rows, and most none at all."""
    rng = np.random.default_rng(24)
    new = [0, 1, 0, 0, 9, 0, 0, 2, 0, 0, 0, 0]
    c = Case(rng, dtype, 1, [5, 700, 0, 3, 1500, 0, 9, 64, 0, 1, 2, 3], new)
    c.fill(upto=c.begin + c.new)
    run_attention(c, 8)


def test_many_sequences():
    """1500 decode rows: several rounds of the plan's sums and of the append's look-ups."""
    rng = np.random.default_rng(25)
    B = 1500
    c = Case(rng, kv8.BF16, 1, rng.integers(0, 40, B), [1] * B)
    c.fill()
    k, v = c.new_kv(spread=3)
    mc.mc_kv8_append(c.desc, 0, dev(k), dev(v), *c.batch())
    c.oracle_append(k, v)
    c.same()
    c.args_begin, c.args_new = c.begin, c.new
    q = normal_bits(rng, (B, 4, 128), kv8.BF16)
    out, lse, _ = attend(c, dev(q).view(torch.bfloat16), 4)
    check_attention(c, q, 4, out, lse)


@pytest.mark.parametrize("new", [1, 40])
def test_pages_beyond_4_gib(new):
    """The same sequence on low pages of a small pool and on pages past 2^32 bytes of a large one: the same bits."""
    rng = np.random.default_rng(26)
    heads, pages = 8, 140000
    c = Case(rng, kv8.BF16, heads, [200], [new])
    c.fill()
    n = len(c.tables[0])
    high = (pages - 1 - rng.permutation(3 * n)[:n]).astype(np.int32)
    assert int(high.min()) * heads * 4096 > 1 << 32
    codes = torch.empty(pages * heads * 4096, dtype=torch.uint8, device=DEV)
    scales = torch.empty((pages, heads, 2), device=DEV)
    big = mc.pool8_desc(codes, scales, 1, pages, heads, kv8.BF16)
    buf = torch.empty(n * heads * 4104, dtype=torch.uint8, device=DEV)
    low_t, high_t = dev(c.tables[0]), dev(high)
    mc.mc_kv8_pack_range(c.desc, 0, 1, low_t, n, 0, 16 * n, buf)
    mc.mc_kv8_unpack_range(big, 0, 1, high_t, n, 0, 16 * n, buf)
    k, v = c.new_kv(spread=3)
    q = dev(normal_bits(rng, (new, 32, 128), kv8.BF16)).view(torch.bfloat16)
    args = c.batch()
    mc.mc_kv8_append(c.desc, 0, dev(k), dev(v), *args)
    low = attend(c, q, 32)
    c.desc, c.args = big, args[:4] + [high_t] + args[5:]
    mc.mc_kv8_append(big, 0, dev(k), dev(v), *c.args)
    got = attend(c, q, 32)
    assert torch.equal(low[0], got[0]) and torch.equal(low[1], got[1])
    pool = torch.zeros((1, n, 2, heads, 16, 128), dtype=torch.bfloat16, device=DEV)
    d16, ident = mc.pool_desc(pool, 1, n, heads, kv8.BF16), torch.arange(n, dtype=torch.int32, device=DEV)
    back = torch.empty_like(buf)
    mc.mc_kv8_pack_range(big, 0, 1, high_t, n, 0, 16 * n, buf)
    mc.mc_kv8_restore_range(big, d16, 0, 1, high_t, n, ident, n, 0, 200 + new)
    mc.mc_kv8_copy_page(big, 0, 1, int(high[0]), 3)
    mc.mc_kv8_compress_range(d16, big, 0, 1, ident, n, high_t, n, 0, 200)
    mc.mc_kv8_pack_range(big, 0, 1, high_t, n, 0, 16 * n, back)
    page = heads * 4096
    assert torch.equal(codes[3 * page:4 * page], buf[:page])
    # whole pages of the 200 tokens: rounding what was rounded changes nothing (a scale may only be a smaller one)
    at = codes.view(pages, 2, heads, 2048)[high_t.long()[:12]].view(torch.float8_e4m3fn).float()
    x = at * scales[high_t.long()[:12]].transpose(1, 2)[..., None]
    k16 = x[:, 0].view(12, heads, 16, 128)
    assert torch.equal(k16, pool[0, :12, 0].float())


def test_begins_out_of_range_are_left_out():
    """At planning time, and when they change behind a plan."""
    rng = np.random.default_rng(27)
    c = Case(rng, kv8.BF16, 2, [40, 50], [1, 20])
    c.fill(upto=c.begin + c.new)
    q = dev(normal_bits(rng, (21, 8, 128), kv8.BF16)).view(torch.bfloat16)
    for begin in ([40, 2 ** 31 - 1], [2 ** 31 - 1, -1], [-2 ** 31, 1 << 30]):
        c.batch()
        size = mc.mc_attn8_workspace_size(2, 21, 8, 2)
        ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
        out = torch.full((21, 8, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
        lse = torch.full((21, 8), float("nan"), device=DEV)
        mc.mc_attn8_plan(c.desc, 8, *c.args, ws, size)
        c.args[3] = dev(np.array(begin, np.int32))
        mc.mc_prefix_prefill_attn8(c.desc, 0, q, 8, *c.args, 0.0, out, lse, ws, size)
        good = begin[0] == 40
        assert torch.isnan(lse[1:]).all() and torch.isnan(lse[0]).any() != good and torch.isnan(out[1:]).all()
        mc.mc_attn8_plan(c.desc, 8, *c.args, ws, size)
        with pytest.raises(mc.McError):
            mc.mc_attn8_plan_check(ws)
        mc.mc_prefix_prefill_attn8(c.desc, 0, q, 8, *c.args, 0.0, out, lse, ws, size)
        assert torch.isnan(lse[1:]).all()


def test_a_plan_of_another_batch_is_refused():
    rng = np.random.default_rng(11)
    c = Case(rng, kv8.BF16, 2, [40], [3])
    c.fill(upto=c.begin + c.new)
    c.batch()
    q = dev(normal_bits(rng, (3, 8, 128), kv8.BF16)).view(torch.bfloat16)
    size = mc.mc_attn8_workspace_size(1, 3, 8, 2)
    ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
    out, lse = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((3, 8), device=DEV)
    mc.mc_attn8_plan(c.desc, 4, *c.args, ws, size)
    mc.mc_prefix_prefill_attn8(c.desc, 0, q, 8, *c.args, 0.0, out, lse, ws, size)
    assert not out.any() and not lse.any()
    ws.zero_()
    mc.mc_prefix_prefill_attn8(c.desc, 0, q, 8, *c.args, 0.0, out, lse, ws, size)
    assert not out.any()
    with pytest.raises(mc.McError):
        mc.mc_attn8_plan_check(ws)


@pytest.mark.parametrize("ctx", [[10, 900, 63], [5000]])
def test_plan_ahead_serves_later_steps(ctx):
    """One plan, 70 tokens ahead; begin grows step by step, past page and tile borders."""
    rng = np.random.default_rng(12)
    ctx = np.array(ctx)
    c = Case(rng, kv8.BF16, 2, ctx, [71] * len(ctx))
    c.fill(upto=ctx + 71)
    B = len(ctx)
    c.batch(ctx, [1] * B)
    size = mc.mc_attn8_workspace_size(B, B, 8, 2)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    mc.mc_attn8_plan_ahead(c.desc, 8, *c.args, 70, ws, size)
    mc.mc_attn8_plan_check(ws)
    for step in (0, 1, 33, 70):
        c.args[3].copy_(torch.from_numpy((ctx + step).astype(np.int32)))
        q = normal_bits(rng, (B, 8, 128), kv8.BF16)
        out = torch.zeros((B, 8, 128), dtype=torch.bfloat16, device=DEV)
        lse = torch.zeros((B, 8), device=DEV)
        mc.mc_prefix_prefill_attn8(c.desc, 0, dev(q).view(torch.bfloat16), 8, *c.args, 0.0, out, lse, ws, size)
        c.args_begin, c.args_new = ctx + step, [1] * B
        check_attention(c, q, 8, out, lse)
    mc.mc_attn8_plan_ahead(c.desc, 8, *c.args, 17, ws, size)         # a page more than the tables have
    with pytest.raises(mc.McError):
        mc.mc_attn8_plan_check(ws)


def test_the_same_call_gives_the_same_bits():
    rng = np.random.default_rng(13)
    c = Case(rng, kv8.BF16, 2, [4000, 100, 2000], [1, 1, 300])
    c.fill(upto=c.begin + c.new)
    c.batch()
    q = dev(normal_bits(rng, (302, 8, 128), kv8.BF16)).view(torch.bfloat16)
    first = attend(c, q, 8)
    for _ in range(4):
        again = attend(c, q, 8)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# --------------------------------------------- conversion, transfer, forks ---
@BOTH
@pytest.mark.parametrize("heads, s0, s1", [(1, 0, 1), (2, 0, 16), (3, 16, 47), (8, 32, 200), (5, 0, 333)])
def test_compress(dtype, heads, s0, s1):
    rng = np.random.default_rng(14)
    L, n = 3, -(-s1 // 16)
    c = Case(rng, dtype, heads, [0], [s1], layers=L)
    pool = normal_bits(rng, (L * (n + 2), 2, heads, 16, 128), dtype, spread=5).reshape(L, n + 2, 2, heads, 16, 128)
    pages = rng.permutation(n + 2)[:n].astype(np.int32)
    t = dev(pool)
    d16 = mc.pool_desc(t, L, n + 2, heads, dtype)
    mc.mc_kv8_compress_range(d16, c.desc, 1, L, dev(pages), n, dev(c.tables[0]), n, s0, s1)
    for layer in range(1, L):
        k, v = (pool[layer, pages, kv].transpose(0, 2, 1, 3).reshape(-1, heads, 128) for kv in (0, 1))
        c.o.append(layer, k[s0:s1], v[s0:s1], s0, c.tables[0])
    c.same()
    assert np.array_equal(t.cpu().numpy().view(np.uint16).reshape(pool.shape), pool)


@BOTH
@pytest.mark.parametrize("heads, s0, s1", [(1, 0, 1), (2, 5, 16), (3, 17, 47), (8, 31, 200), (5, 0, 333)])
def test_restore(dtype, heads, s0, s1):
    rng = np.random.default_rng(15)
    L, n = 3, -(-s1 // 16)
    c = Case(rng, dtype, heads, [0], [s1], layers=L)
    c.o.codes[:] = rng.integers(0, 256, c.o.codes.shape)
    lo, hi = kv8.LIMITS[dtype]
    c.o.k[:] = rng.integers(max(lo, -30), min(hi, 30) - (hi < 30), c.o.k.shape)
    c.upload()
    was = normal_bits(rng, (L * (n + 2), 2, heads, 16, 128), dtype).reshape(L, n + 2, 2, heads, 16, 128)
    pages = rng.permutation(n + 2)[:n].astype(np.int32)
    t = dev(was)
    d16 = mc.pool_desc(t, L, n + 2, heads, dtype)
    mc.mc_kv8_restore_range(c.desc, d16, 0, 2, dev(c.tables[0]), n, dev(pages), n, s0, s1)
    got = t.cpu().numpy().view(np.uint16).reshape(was.shape)
    want = kv8.decode16(was, dtype)
    for layer in range(2):
        for kv, x in enumerate(c.o.values(layer, c.tables[0], s1)):
            for pos in range(s0, s1):
                want[layer, pages[pos // 16], kv, :, pos % 16] = x[:, pos]
    assert np.array_equal(kv8.decode16(got, dtype), want, equal_nan=True)
    c.same()


def test_conversion_leaves_out_pages_the_pools_do_not_have():
    rng = np.random.default_rng(16)
    c = Case(rng, kv8.BF16, 2, [0], [64])
    pool = torch.zeros((1, 6, 2, 2, 16, 128), dtype=torch.bfloat16, device=DEV)
    count = torch.zeros(1, dtype=torch.int32, device=DEV)
    d16 = mc.pool_desc(pool, 1, 6, 2, kv8.BF16, skipped=count)
    bad16, bad8 = dev(np.array([0, 6, 2, 3], np.int32)), dev(np.array([c.tables[0][0], 1, -1, c.tables[0][3]], np.int32))
    mc.mc_kv8_compress_range(d16, c.desc, 0, 1, bad16, 4, bad8, 4, 0, 64)
    for i in (0, 3):
        c.o.append(0, np.zeros((16, 2, 128), np.uint16), np.zeros((16, 2, 128), np.uint16), 16 * i, c.tables[0])
    c.same()
    assert c.skipped.item() == 2 and count.item() == 0
    mc.mc_kv8_restore_range(c.desc, d16, 0, 1, bad8, 4, bad16, 4, 3, 64)
    assert mc.mc_kv_copy_check(d16) == (mc.MC_ERR_RANGE, 2) and not pool.any()


@pytest.mark.parametrize("heads, layers, s0, s1", [(1, 1, 0, 1), (2, 3, 16, 47), (8, 2, 32, 200), (11, 2, 0, 333)])
def test_pack_and_unpack_move_whole_pages(heads, layers, s0, s1):
    rng = np.random.default_rng(17)
    n, first = -(-s1 // 16), s0 // 16
    c = Case(rng, kv8.F16, heads, [0], [s1], layers=layers + 1)
    c.o.codes[:] = rng.integers(0, 256, c.o.codes.shape)
    c.o.k[:] = rng.integers(-15, 9, c.o.k.shape)
    c.upload()
    size = layers * (n - first) * heads * 4104
    buf = torch.full((size + 64,), 0xab, dtype=torch.uint8, device=DEV)
    mc.mc_kv8_pack_range(c.desc, 1, layers + 1, dev(c.tables[0]), n, s0, s1, buf)
    raw, scales = c.o.raw()
    moved = c.tables[0][first:]
    want = np.concatenate([raw[1:, moved].ravel(), scales[1:, moved].ravel().view(np.uint8)])
    got = buf.cpu().numpy()
    assert np.array_equal(got[:size], want) and np.all(got[size:] == 0xab)
    c.same()
    r = Case(rng, kv8.F16, heads, [0], [s1], layers=layers)          # the receiver
    mc.mc_kv8_unpack_range(r.desc, 0, layers, dev(r.tables[0]), n, s0, s1, buf)
    r.o.codes[:, r.tables[0][first:]] = c.o.codes[1:, moved]
    r.o.k[:, r.tables[0][first:]] = c.o.k[1:, moved]
    r.same()
    bad = r.tables[0].copy()
    bad[-1] = r.num_pages
    mc.mc_kv8_unpack_range(r.desc, 0, layers, dev(bad), n, s0, s1, buf)
    mc.mc_kv8_pack_range(r.desc, 0, layers, dev(bad), n, s0, s1, buf)
    r.same()
    assert mc.mc_kv8_copy_check(r.desc) == (mc.MC_ERR_RANGE, 2)


def test_copy_page():
    rng = np.random.default_rng(18)
    c = Case(rng, kv8.BF16, 3, [0], [100], layers=4)
    c.o.codes[:] = rng.integers(0, 256, c.o.codes.shape)
    c.o.k[:] = rng.integers(-20, 20, c.o.k.shape)
    c.upload()
    mc.mc_kv8_copy_page(c.desc, 1, 3, 2, 7)
    c.o.codes[1:3, 7], c.o.k[1:3, 7] = c.o.codes[1:3, 2], c.o.k[1:3, 2]
    c.same()


# ------------------------------------------------------- as they are used ----
def test_a_prompt_from_one_engine_to_another():
    """A cached prompt leaves a 16-bit pool for the 8-bit one; new tokens are appended and attend over it; the sequence
    is forked and both go on, one token at a time; its pages go to another engine, which attends to the same bits."""
    rng = np.random.default_rng(19)
    L, heads, hq, cached, n = 2, 2, 8, 100, 37
    alloc = mc.mc_kv_allocator_create(40)
    table = np.array(mc.mc_kv_alloc_pages(alloc, 9), np.int32)
    c = Case(rng, kv8.BF16, heads, [cached], [n], layers=L, spare=40 - 9, tables=[table])
    pool = normal_bits(rng, (L * 9, 2, heads, 16, 128), kv8.BF16).reshape(L, 9, 2, heads, 16, 128)
    t16 = dev(pool)
    d16 = mc.pool_desc(t16, L, 9, heads, kv8.BF16)
    ident = dev(np.arange(9, dtype=np.int32))
    mc.mc_kv8_compress_range(d16, c.desc, 0, L, ident, 9, dev(table), 9, 0, cached)
    c.batch()
    for layer in range(L):
        old = [pool[layer, :, kv].transpose(0, 2, 1, 3).reshape(-1, heads, 128)[:cached] for kv in (0, 1)]
        c.o.append(layer, *old, 0, table)
        k, v = c.new_kv()
        mc.mc_kv8_append(c.desc, layer, dev(k), dev(v), *c.args)
        c.oracle_append(k, v, layer)
        q = normal_bits(rng, (n, hq, 128), kv8.BF16)
        out, lse, _ = attend(c, dev(q).view(torch.bfloat16), hq, layer=layer)
        c.args_begin, c.args_new = c.begin, c.new
        check_attention(c, q, hq, out, lse, layer=layer)
    c.same()
    # fork at 137 tokens: page 8 holds nine of them
    child, (src, dst, slots) = mc.mc_kv_fork_sequence(alloc, table.tolist(), cached + n)
    assert slots == 9
    mc.mc_kv8_copy_page(c.desc, 0, L, src, dst)
    c.o.codes[:, dst], c.o.k[:, dst] = c.o.codes[:, src], c.o.k[:, src]
    both = Case(rng, kv8.BF16, heads, [cached + n] * 2, [1, 1], layers=L, tables=[table, np.array(child, np.int32)])
    both.o, both.num_pages = c.o, c.num_pages
    both.codes, both.scales, both.desc = c.codes, c.scales, c.desc
    for step in range(3):
        both.begin = np.array([cached + n + step] * 2)
        both.args_begin, both.args_new = both.begin, both.new
        both.batch()
        for layer in range(L):
            k, v = both.new_kv(spread=3)
            mc.mc_kv8_append(c.desc, layer, dev(k), dev(v), *both.args)
            both.oracle_append(k, v, layer)
            q = normal_bits(rng, (2, hq, 128), kv8.BF16)
            out, lse, _ = attend(both, dev(q).view(torch.bfloat16), hq, layer=layer)
            check_attention(both, q, hq, out, lse, layer=layer)
    both.same()
    # the sequence as it was after the prompt, on another engine
    r = Case(rng, kv8.BF16, heads, [cached], [n], layers=L)
    buf = torch.empty(L * 9 * heads * 4104, dtype=torch.uint8, device=DEV)
    mc.mc_kv8_pack_range(c.desc, 0, L, dev(table), 9, 0, cached + n, buf)
    mc.mc_kv8_unpack_range(r.desc, 0, L, dev(r.tables[0]), 9, 0, cached + n, buf)
    r.o.codes[:, r.tables[0]], r.o.k[:, r.tables[0]] = c.o.codes[:, table], c.o.k[:, table]
    r.same()
    r.batch()
    c.batch()
    for layer in range(L):
        q = dev(normal_bits(rng, (n, hq, 128), kv8.BF16)).view(torch.bfloat16)
        there, here = attend(r, q, hq, layer=layer), attend(c, q, hq, layer=layer)
        assert torch.equal(there[0], here[0]) and torch.equal(there[1], here[1])
    mc.mc_kv_allocator_destroy(alloc)


@BOTH
@pytest.mark.parametrize("new", [1, 4, 90])
def test_scores_are_sums_in_32_bits(dtype, new):
    """Two products of +-256 that cancel, and 126 of j 2^-9, |j| <= 15: every sum of some of them is a multiple of 2^-9
    below 2^10, so exact in fp32 in whatever order, while a sum that drops what is 2^-13 of its largest term would lose
    most of the score.  A score is then below 4, and what is left is the roundings of the scaled score, the exponential
    and the logarithm (a few 2^-24 of at most 8) and of the sum (one 2^-24 for each key, in the worst order)."""
    rng = np.random.default_rng(23)
    c = Case(rng, dtype, 2, [150], [new])
    n = 150 + new
    t = TYPES[dtype]
    bits = lambda x: torch.from_numpy(x).to(t).view(torch.int16).numpy().view(np.uint16)
    k = rng.integers(1, 16, (n, 2, 128)) * 2.0 ** -9
    k[:, :, 0], k[:, :, 1] = 2.0, -2.0
    c.o.append(0, bits(k), normal_bits(rng, (n, 2, 128), dtype), 0, c.tables[0])
    c.upload()
    c.args_begin, c.args_new = c.begin, c.new
    c.batch()
    q = rng.choice([-1.0, 1.0, 1.0], (new, 8, 128))
    q[:, :, 0], q[:, :, 1] = 128.0, 128.0
    _, lse, _ = attend(c, dev(bits(q)).view(t), 8)
    s = np.einsum("qhd,khd->qhk", q, np.repeat(k, 4, 1)) / np.sqrt(128.0)
    s = np.where(np.arange(n) <= 150 + np.arange(new)[:, None, None], s, -np.inf)
    want = np.log(np.exp(s).sum(-1))
    err = np.abs(lse.double().cpu().numpy() - want).max()
    assert err <= (n + 64) * 2.0 ** -24, err


def test_as_exact_as_the_16_bit_path_on_the_same_numbers():
    """The 8-bit cache restored to a 16-bit pool holds the same K and V: both attentions agree within two roundings."""
    rng = np.random.default_rng(20)
    c = Case(rng, kv8.BF16, 2, [300], [60])
    c.fill(upto=c.begin + c.new)
    c.batch()
    n = len(c.tables[0])
    pool = torch.zeros((1, n, 2, 2, 16, 128), dtype=torch.bfloat16, device=DEV)
    d16 = mc.pool_desc(pool, 1, n, 2, kv8.BF16)
    ident = torch.arange(n, dtype=torch.int32, device=DEV)
    mc.mc_kv8_restore_range(c.desc, d16, 0, 1, dev(c.tables[0]), n, ident, n, 0, 360)
    q = normal_bits(rng, (60, 8, 128), kv8.BF16)
    dq = dev(q).view(torch.bfloat16)
    out, lse, _ = attend(c, dq, 8)
    size = mc.mc_attn_workspace_size(1, 60, 8, 2)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    args = [1, 60, cu([60]), dev(np.array([300], np.int32)), ident, cu([n])]
    mc.mc_attn_plan(d16, 8, *args, ws, size)
    out16, lse16 = torch.zeros_like(out), torch.zeros_like(lse)
    mc.mc_prefix_prefill_attn(d16, 0, dq, 8, *args, 0.0, out16, lse16, ws, size)
    want = kv8.attention(c.o, 0, c.tables[0], q, 300)
    for o, l in ((out, lse), (out16, lse16)):
        close(o.double().cpu().numpy(), l.double().cpu().numpy(), want, kv8.BF16, 360)


def test_captured_steps_replay():
    """Plan, append and attention of a decode step and a range captured into a graph and replayed with other tokens and
    lengths, eager work between the replays."""
    rng = np.random.default_rng(21)
    lens = np.array([200, 1000, 37])
    c = Case(rng, kv8.BF16, 2, lens, [10, 60, 25])
    c.fill()
    new = np.array([1, 20, 1])
    B, tq = 3, 22
    c.batch(lens, new)
    size = mc.mc_attn8_workspace_size(B, tq, 8, 2)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    q, k, v = (torch.zeros((tq, h, 128), dtype=torch.bfloat16, device=DEV) for h in (8, 2, 2))
    out, lse = torch.zeros_like(q), torch.zeros((tq, 8), device=DEV)

    def step():
        mc.mc_attn8_plan(c.desc, 8, *c.args, ws, size)
        mc.mc_kv8_append(c.desc, 0, k, v, *c.args)
        mc.mc_prefix_prefill_attn8(c.desc, 0, q, 8, *c.args, 0.0, out, lse, ws, size)
    step()
    torch.cuda.synchronize()
    raw, scales = c.o.raw()
    c.codes.copy_(torch.from_numpy(raw))
    c.scales.copy_(torch.from_numpy(scales))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    begin = lens.copy()
    for i in range(4):
        bits = [normal_bits(rng, (tq, h, 128), kv8.BF16) for h in (8, 2, 2)]
        for t, b in zip((q, k, v), bits):
            t.view(torch.int16).copy_(torch.from_numpy(b.view(np.int16)))
        c.args[3].copy_(torch.from_numpy(begin.astype(np.int32)))
        if i == 2:
            step()                     # the same work eagerly, on the same buffers
        else:
            g.replay()
        torch.cuda.synchronize()
        c.begin, c.new = begin, new
        c.oracle_append(bits[1], bits[2])
        c.same()
        c.args_begin, c.args_new = begin, new
        check_attention(c, bits[0], 8, out, lse)
        begin = begin + np.array([1, 13, 1])           # (the range is written again from its 14th token on)


def test_on_another_stream():
    rng = np.random.default_rng(22)
    c = Case(rng, kv8.BF16, 2, [500], [3])
    c.fill()
    k, v = c.new_kv()
    c.batch()
    c.args_begin, c.args_new = c.begin, c.new
    q = normal_bits(rng, (3, 8, 128), kv8.BF16)
    dk, dv, dq = dev(k), dev(v), dev(q).view(torch.bfloat16)
    size = mc.mc_attn8_workspace_size(1, 3, 8, 2)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    out, lse = torch.zeros_like(dq), torch.zeros((3, 8), device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    mc.mc_attn8_plan(c.desc, 8, *c.args, ws, size, stream=side)
    mc.mc_kv8_append(c.desc, 0, dk, dv, *c.args, stream=side)
    mc.mc_prefix_prefill_attn8(c.desc, 0, dq, 8, *c.args, 0.0, out, lse, ws, size, stream=side.cuda_stream)
    side.synchronize()
    c.oracle_append(k, v)
    c.same()
    check_attention(c, q, 8, out, lse)
