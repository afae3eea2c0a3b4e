"""The token calls (include/az_tokens.h) at the ends of what they allow: slices of a row that hold nothing, scales and sizes near
the limits of their types.  Statements in 64 bits and tolerances as in test_gpu_tokens.py."""
import ctypes
import math
import os
import subprocess
import sys
import threading
import time

import pytest
import torch

from test_gpu_tokens import (BF16, F16, F32, TYPES, U, az, check_logits, check_product, clean_status, dequantised, gen, half_step,  # noqa: F401
                             make_rules, operand, padded, reference, smallest, up)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def release_memory():
    """Some tests hold tens of gigabytes; the next ones may run in other processes."""
    yield
    torch.cuda.empty_cache()


# ---- logits: CTAs of a cluster whose share of the row holds nothing ------------------------------------------

# what the few tokens that are left have for logits, and the temperature
LOW_ROWS = [(-1.0, 0.01), (-5.0, 0.05), (-10.0, 0.05), (-9.0, 0.1), (-45.0, 0.5), (-100.0, 1.0), (-200.0, 1.0), (30.0, 0.02), (-0.01, 1.0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1858, 5000, 40000, 100277, 131072, 200003])
@pytest.mark.parametrize("closed_by", ["mask", "logits", "both", "lowest"])
@pytest.mark.parametrize("tokens", [1, 3])
def test_low_logits_beside_slices_that_hold_nothing(az, dtype, vocab, closed_by, tokens):
    """A strict grammar at a low temperature: a few tokens with low logits, nothing in most CTAs' shares of the row."""
    rows = len(LOW_ROWS)
    level, heat = (torch.tensor(v, device="cuda", dtype=F32) for v in zip(*LOW_ROWS))
    place = torch.tensor([vocab // 3, vocab // 3 + 1, vocab - 1][:tokens], device="cuda")
    spread = torch.tensor([0.0, -0.5, -1.0][:tokens], device="cuda")
    kept = (level[:, None] + spread * heat[:, None]).to(dtype)
    closed = {"mask": 0.5, "lowest": torch.finfo(dtype).min}.get(closed_by, -math.inf)
    logits = torch.full((rows, vocab), closed, device="cuda", dtype=dtype)
    logits[:, place] = kept
    rules = {"temperature": heat}
    if closed_by in ("mask", "both"):
        bits = torch.zeros(-(-vocab // 32) * 32, dtype=torch.int64, device="cuda")
        bits[place] = 1
        words = (bits.view(-1, 32) << torch.arange(32, device="cuda")).sum(1)
        rules["allowed"] = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()
    x = (kept.double() - kept.double().amax(1, keepdim=True)) / heat.double()[:, None]
    total = x.exp().sum(1, keepdim=True)
    want = x.exp() / total
    rel = (12 * kept.double().abs().amax(1, keepdim=True) / heat.double()[:, None] + 5 * x.abs() + 120) * U
    rest = torch.ones(vocab, dtype=torch.bool, device="cuda")
    rest[place] = False
    for kind in {dtype, F32}:
        probs = torch.full((rows, vocab), -1.0, device="cuda", dtype=kind)
        best = torch.empty(rows, dtype=torch.int32, device="cuda")
        logprob = torch.empty(rows, device="cuda")
        az.az_token_probs(logits, probs, best, logprob, **rules)
        assert (probs[:, rest] == 0).all()
        assert ((probs[:, place].double() - want).abs() <= (rel + half_step(kind)) * want + smallest(kind)).all()
        top = kept.double().argmax(1)
        assert torch.equal(best.long(), place[top])
        assert ((logprob.double() + total.log()[:, 0]).abs() <= 2 * rel.amax(1) + 1e-7).all()


def test_every_slice_but_one_holds_nothing_wherever_it_is(az):
    """One token left, in each chunk of the row in turn."""
    vocab, rows = 131072, 512
    place = torch.arange(rows, device="cuda") * 256 + 17
    logits = torch.full((rows, vocab), -math.inf, device="cuda", dtype=BF16)
    logits[torch.arange(rows, device="cuda"), place] = -300.0
    probs = torch.empty_like(logits)
    best = torch.empty(rows, dtype=torch.int32, device="cuda")
    logprob = torch.empty(rows, device="cuda")
    az.az_token_probs(logits, probs, best, logprob)
    assert torch.equal(best.long(), place) and (logprob == 0).all()
    assert (probs != 0).sum() == rows and (probs[torch.arange(rows, device="cuda"), place] == 1).all()


# ---- indices near 2^31 ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("twice", [False, True])
def test_bias_lists_that_end_at_the_last_index(az, twice):
    """Lists at the end of 2^31 - 1 entries give what the same lists give in a short buffer."""
    count = 2 ** 31 - 1
    lengths = [600, 0, 700, 1, 31]
    total = sum(lengths)
    short = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()
    long_tokens = torch.zeros(count, dtype=torch.int32, device="cuda")
    long_values = torch.full((count,), 100.0, device="cuda")
    for vocab in (1858, 9000, 131072):
        g = gen(vocab)
        tokens = torch.cat([torch.randperm(vocab, generator=g, device="cuda")[:n] for n in lengths]).int()
        if twice:
            tokens[5:600:7] = tokens[3]
            tokens[total - 1] = tokens[total - 2]
        values = torch.randn(total, generator=g, device="cuda")
        long_tokens[count - total:] = tokens
        long_values[count - total:] = values
        logits = torch.randn(len(lengths), vocab, generator=g, device="cuda")
        want, got = torch.empty_like(logits), torch.empty_like(logits)
        az.az_adjust_logits(logits, want, bias_offsets=short, bias_tokens=tokens, bias_values=values)
        az.az_adjust_logits(logits, got, bias_offsets=short + (count - total), bias_tokens=long_tokens, bias_values=long_values)
        assert torch.equal(want, got)
        exact = logits.double()
        if not twice:
            owner = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda"))
            exact = exact.index_put((owner, tokens.long()), values.double(), accumulate=True)
            assert ((got.double() - exact).abs() <= U * exact.abs()).all()
    # offsets beyond the buffer are clamped to it: lists that hold nothing
    none = torch.full((len(lengths) + 1,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    az.az_adjust_logits(logits, got, bias_offsets=none, bias_tokens=long_tokens, bias_values=long_values)
    assert torch.equal(got, logits)


def test_the_largest_number_of_rows(az):
    """2^31 - 1 rows of one token: the step behind the last row leaves 31 bits, and nothing in front of the buffers is touched."""
    rows, guard = 2 ** 31 - 1, 1 << 20
    flat = torch.full((guard + rows + guard,), 3.0, device="cuda", dtype=BF16)
    logits = flat[guard:guard + rows].view(rows, 1)
    nothing, all_of_it = (torch.full((1,), v, dtype=torch.int32, device="cuda") for v in (0, -1))
    best = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    logits[::5] = -math.inf
    az.az_token_probs(logits, best=best, allowed=all_of_it)
    assert (best[::5] == -1).all()
    best[::5] = 0
    assert (best == 0).all()
    az.az_adjust_logits(logits, logits, allowed=nothing)
    assert (flat[guard:guard + rows] == -math.inf).all()
    assert (flat[:guard] == 3.0).all() and (flat[guard + rows:] == 3.0).all()
    az.az_token_probs(logits, logits, best)                   # rows that hold nothing, in place
    assert (flat[guard:guard + rows] == 0).all() and (best == -1).all()
    assert (flat[:guard] == 3.0).all() and (flat[guard + rows:] == 3.0).all()


# ---- the status word ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("part", [0, 1])
def test_a_wait_that_runs_out_is_reported_once(az, part):
    az.az_selftest_tokens_timeout(part)
    word = az.az_tokens_status()
    assert word != 0 and az.az_tokens_status() == 0
    raw = ctypes.c_uint32(0)
    az.az_selftest_tokens_timeout(part)
    stream = torch.cuda.current_stream().cuda_stream
    assert az._lib.az_tokens_status(stream, ctypes.byref(raw)) == az.AZ_ERR_DEVICE_TIMEOUT and raw.value == word
    assert az._lib.az_tokens_status(stream, ctypes.byref(raw)) == az.AZ_OK and raw.value == 0
    x, y = torch.ones(3, 5000, device="cuda"), torch.empty(3, 5000, device="cuda")
    az.az_token_probs(x, y)                                   # the device still works
    assert ((y.double() - 1 / 5000).abs() <= 120 * U / 5000).all()


@pytest.mark.parametrize("part", [0, 1])
def test_no_report_is_lost_between_streams(az, part):
    """One thread reads the status without a pause while kernels on another stream raise it: every one of them is reported."""
    reading, raising = torch.cuda.Stream(), torch.cuda.Stream()
    reports, stop, failed = [0], threading.Event(), []

    def read():
        try:
            while not stop.is_set():
                if az.az_tokens_status(reading):
                    reports[0] += 1
        except Exception as e:
            failed.append(e)

    reader = threading.Thread(target=read)
    reader.start()
    try:
        for i in range(200):
            before = reports[0]
            az.az_selftest_tokens_timeout(part, raising)
            raising.synchronize()
            limit = time.monotonic() + 5
            while reports[0] == before and time.monotonic() < limit and not failed:
                time.sleep(0.0002)
            assert not failed and reports[0] > before, i
    finally:
        stop.set()
        reader.join()
    assert az.az_tokens_status() == 0
    with pytest.raises(az.AzError):
        az.az_selftest_tokens_timeout(2)


# ---- products of scales beyond float32's range -----------------------------------------------------------------

@pytest.mark.parametrize("m,n,k", [(1, 130, 512), (20, 20001, 300), (40, 300, 3000), (100, 300, 512), (100, 20001, 300), (400, 14100, 400)])
def test_products_of_scales_beyond_float32(az, m, n, k):
    """A pair whose product overflows reaches its row and its 128 columns, no others; products below 2^-126 keep fewer bits."""
    g = gen(m + n + k)
    codes = [torch.randint(0, 0x7f, (rows, up(k, 16)), generator=g, device="cuda", dtype=torch.uint8)[:, :k] for rows in (m, n)]
    kb, nb = -(-k // 128), -(-n // 128)
    sa = 2.0 ** -80 * (1 + torch.rand(m, kb, generator=g, device="cuda"))
    sb = 2.0 ** -60 * (1 + torch.rand(nb, kb, generator=g, device="cuda"))
    out = torch.empty(m, n, device="cuda")
    az.az_block_matmul(codes[0], sa, codes[1], sb, out)
    x, w = dequantised(codes[0], sa, 1), dequantised(codes[1], sb, 128)
    want = x @ w.t()                                          # (all terms are positive: also the sum of magnitudes)
    # a block's factor is off by up to 2^-150 there, its sum is at most 128 x 448 x 448 < 2^25
    assert ((out.double() - want).abs() <= (256 + k / 128 + 12) * U * want + kb * 2.0 ** -125 + smallest(F32)).all()
    row, block = m // 2, nb - 1
    sa[row, 0], sb[block, 0] = 2.0 ** 66, 2.0 ** 66
    az.az_block_matmul(codes[0], sa, codes[1], sb, out)
    assert not out[row, block * 128:].isfinite().any()
    out[row, block * 128:] = 0
    assert out.isfinite().all()


# ---- rows of the product that are written two elements at a time -------------------------------------------------

@pytest.mark.parametrize("m,n,k", [(129, 14402, 300), (300, 15002, 400), (369, 20006, 577), (384, 14340, 136), (128, 15002, 300)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_every_alignment_hold_the_same_bits(az, m, n, k, dtype):
    """The form of the kernel goes by the rows' alignment too, the order of a sum does not."""
    a, sa = operand(m, k, 1, 1)
    b, sb = operand(n, k, 128, 2)
    v = torch.randn(n, generator=gen(3), device="cuda")
    outs = []
    for stride, offset in ((up(n, 8), 0), (n, 0), (n + 2, 2), (n + 1, 1)):
        flat, out = padded(m, n, stride, dtype, -7.0, offset)
        az.az_block_matmul(a, sa, b, sb, out, bias=v)
        rest = flat[offset:offset + m * stride].view(m, stride)[:, n:]
        assert (rest == -7.0).all() and (flat[:offset] == -7.0).all() and (flat[offset + m * stride:] == -7.0).all()
        outs.append(out)
    assert all(torch.equal(outs[0], out) for out in outs)
    check_product(az, m, n, k, dtype, True, 5)


# ---- parameters at the ends of their types ---------------------------------------------------------------------

@pytest.mark.parametrize("vocab", [1858, 9000, 131072])
def test_the_lowest_and_highest_temperatures(az, vocab):
    heat = torch.tensor([2.0 ** -126, 1e-37, 1e-30, 1.0, 1e30, torch.finfo(F32).max], device="cuda")
    rows = len(heat)
    logits = torch.randn(rows, vocab, generator=gen(vocab), device="cuda") * 3 - 20
    probs, out = torch.empty_like(logits), torch.empty_like(logits)
    best = torch.empty(rows, dtype=torch.int32, device="cuda")
    logprob = torch.empty(rows, device="cuda")
    az.az_token_probs(logits, probs, best, logprob, temperature=heat)
    top = logits.argmax(1)
    assert torch.equal(best.long(), top)
    one = torch.nn.functional.one_hot(top[:3], vocab).to(F32)
    assert torch.equal(probs[:3], one) and (logprob[:3] == 0).all()
    # hot rows: every exponent is 0 up to 1e-29
    assert ((probs[4:].double() * vocab - 1).abs() <= 120 * U).all()
    assert ((logprob[4:].double() + math.log(vocab)).abs() <= 240 * U + 4 * U * math.log(vocab) + 1e-7).all()
    az.az_adjust_logits(logits, out, temperature=heat)
    want = logits.double() / heat.double()[:, None]
    fine = want.abs() < 3e38
    # (1 / T below the normal range: off by 2^-150, under 2^-20 of itself)
    assert ((out.double() - want).abs()[fine] <= (2.0 ** -20 * want.abs() + smallest(F32))[fine]).all()
    assert (out[~fine & (want < -3.5e38)] == -math.inf).all()


@pytest.mark.parametrize("vocab", [1858, 9000, 131072])
def test_tokens_lengths_and_offsets_at_the_ends_of_their_type(az, vocab):
    """Ids outside the vocabulary are skipped and lengths and offsets clamped, be they the least or the greatest 32-bit numbers."""
    low, high = -2 ** 31, 2 ** 31 - 1
    rows, room = 6, 40
    g = gen(vocab)
    tokens = torch.randint(0, vocab, (rows, room), generator=g, device="cuda").int()
    tokens[:, ::3] = torch.tensor([low, -1, vocab, vocab + 7, high - 7, high], device="cuda", dtype=torch.int32)[:, None]
    lengths = torch.tensor([high, low, room, high, 17, room], device="cuda", dtype=torch.int32)
    prompts = torch.tensor([low, high, 5, high, high, -1], device="cuda", dtype=torch.int32)
    names = torch.tensor([low, 3, vocab - 1, vocab, high - 3, high, 8, 5, 9, 11], device="cuda", dtype=torch.int32)
    values = torch.randn(len(names), generator=g, device="cuda")
    rules = dict(tokens=tokens, lengths=lengths, prompt_lengths=prompts, repetition=torch.full((rows,), 1.3, device="cuda"),
                 presence=torch.full((rows,), 0.5, device="cuda"), frequency=torch.full((rows,), 0.25, device="cuda"))
    logits = torch.randn(rows, vocab, generator=g, device="cuda") * 4
    plain = dict(rules, bias_offsets=torch.tensor([0, 8, 10, 10, 10, 10, 10], device="cuda", dtype=torch.int32), bias_tokens=names,
                 bias_values=values)
    want = reference(logits, plain)
    check_logits(az, logits, plain, want=want)
    wild = dict(plain, bias_offsets=torch.tensor([low, 8, high, high, low, low, high], device="cuda", dtype=torch.int32))
    # rows 0, 1: as above; row 2: high .. high, 3: high .. low, 4: low .. low: nothing; row 5: all of the list
    want = reference(logits, dict(rules, bias_offsets=torch.tensor([0, 8, 10, 10, 10, 10, 20], device="cuda", dtype=torch.int32),
                                  bias_tokens=torch.cat([names, names]), bias_values=torch.cat([values, values])))
    check_logits(az, logits, wild, want=want)


@pytest.mark.parametrize("wide", [False, True])
def test_the_largest_products(az, wide):
    """2^31 - 256 rows, and as many columns: every output, at its place."""
    most, k = 2 ** 31 - 256, 16
    long, one = torch.full((most, k), 0x38, dtype=torch.uint8, device="cuda"), torch.full((1, k), 0x40, dtype=torch.uint8, device="cuda")     # 1.0 and 2.0
    long[::1000003] = 0x30                                    # 0.5
    step = 128 if wide else 1
    scales = torch.ones((-(-most // step), 1), device="cuda")
    scales[-1] = 4.0
    unit = torch.ones((1, 1), device="cuda")
    out = torch.full((1, most) if wide else (most, 1), -7.0, device="cuda", dtype=BF16)
    if wide:
        az.az_block_matmul(one, unit, long, scales, out)
    else:
        az.az_block_matmul(long, scales, one, unit, out)
    flat = out.view(-1)
    flat[most - step:] /= 4.0
    assert (flat[::1000003] == 16.0).all()
    flat[::1000003] = 32.0
    assert (flat == 32.0).all()


def test_the_largest_number_of_quantised_rows(az):
    rows = 2 ** 31 - 1
    x = torch.full((rows, 1), 2.0, device="cuda", dtype=BF16)
    x[::1000003] = 0.0
    codes = torch.full((rows, 1), 0x55, device="cuda", dtype=torch.uint8)
    scales = torch.full((rows, 1), -7.0, device="cuda")
    az.az_quantise_blocks(x, codes, scales, 1)
    assert (scales[::1000003] == 2.0 ** -126).all() and ((codes[::1000003] & 0x7f) == 0).all()
    scales[::1000003], codes[::1000003] = 2.0 / 448, 0x7e
    assert (scales == 2.0 / 448).all() and (codes == 0x7e).all()
    few = scales[: -(-rows // 128)]
    few.fill_(-7.0)
    az.az_quantise_blocks(x, codes, few, 128)
    assert (few == 2.0 / 448).all() and (codes[1::1000003] == 0x7e).all() and ((codes[::1000003] & 0x7f) == 0).all()


# ---- the quantiser's quotients -----------------------------------------------------------------------------------

def codes_by_definition(x, scale):
    """|x| / scale rounded once to e4m3, as code magnitudes, by comparison with the middles between codes (float64, on the GPU)."""
    grid = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    middle = (grid[1:] + grid[:-1]) / 2
    ratio = x.double().abs() / scale.double()
    low, high = torch.bucketize(ratio, middle), torch.bucketize(ratio, middle, right=True)
    return torch.where(low % 2 == 0, low, high)


@pytest.mark.parametrize("dtype,mantissa", [(F16, 10), (BF16, 7)])
@pytest.mark.parametrize("exponent", ["lowest", "low", "one", "highest"])
def test_every_16_bit_number_under_every_maximum(az, dtype, mantissa, exponent):
    """Each 16-bit magnitude in a block with each mantissa of a maximum: the codes are those of the real quotients."""
    info = torch.finfo(dtype)
    first = {"lowest": 1, "low": (torch.tensor(info.smallest_normal, dtype=dtype).view(torch.int16).item()),
             "one": torch.tensor(1.0, dtype=dtype).view(torch.int16).item(),
             "highest": torch.tensor(info.max, dtype=dtype).view(torch.int16).item() - (1 << mantissa) + 1}[exponent]
    tops = torch.arange(first, first + (1 << mantissa), device="cuda")
    # magnitudes within 2^16 of the maximum: smaller ones have the code 0
    reach = 16 << mantissa
    offsets = torch.arange(-reach, 1 << mantissa, device="cuda")
    per_row = -(-len(offsets) // 127)
    offsets = torch.nn.functional.pad(offsets, (0, per_row * 127 - len(offsets)))
    for some in tops.split(max(1, (1 << 25) // len(offsets))):
        bits = (some[:, None] + offsets).clamp_min(0)
        bits = torch.where(bits > some[:, None], 0, bits).view(len(some), per_row, 127)
        bits = torch.cat([bits, some[:, None, None].expand(-1, per_row, 1)], 2).view(len(some), per_row * 128)
        x = bits.to(torch.int16).view(dtype)
        codes, scales = torch.empty(x.shape, dtype=torch.uint8, device="cuda"), torch.empty(len(some), per_row, device="cuda")
        az.az_quantise_blocks(x, codes, scales, 1)
        top = some.to(torch.int16).view(dtype).double()
        want = torch.maximum((top / 448).float(), torch.tensor(2.0 ** -126, device="cuda"))
        assert (scales == want[:, None]).all()
        assert torch.equal((codes & 0x7f).long(), codes_by_definition(x, want[:, None]))


# ---- probabilities near the end of float32 ---------------------------------------------------------------------

@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(4, 1858), (4, 9000), (4, 40000), (3, 131072), (200, 20000)])
def test_small_probabilities_of_slices_far_below_the_best(az, kind, rows, vocab):
    """Chunks of the row whose best tokens have probabilities from 1 down to nothing: each right to the last number of its type."""
    g = gen(vocab)
    chunk = torch.arange(vocab, device="cuda") // 256
    level = -106 * torch.rand((rows, int(chunk[-1]) + 1), generator=g, device="cuda")
    level[:, 0] = 0.0
    heat = torch.tensor([1.0, 0.05, 0.7, 0.01], device="cuda")[torch.arange(rows, device="cuda") % 4]
    logits = level[:, chunk] - torch.rand((rows, vocab), generator=g, device="cuda")
    for slices in (1, 8):                                     # neighbouring chunks alike: whole slices far below
        some = level[:, (chunk % slices)] - torch.rand((rows, vocab), generator=g, device="cuda") if slices > 1 else logits
        check_logits(az, ((some - 3.0) * heat[:, None]).to(kind), {"temperature": heat}, F32)
        check_logits(az, ((some - 3.0) * heat[:, None]).to(kind), {"temperature": heat}, kind)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [300, 1858, 9001, 40000, 131072])
@pytest.mark.parametrize("rows", [12, 300])
def test_infinities_and_nan_anywhere_in_a_row(az, dtype, vocab, rows):
    """One to three odd values in each row, allowed or not, wherever the row is cut."""
    if rows * vocab > 1 << 24:
        rows = 60
    g = gen(vocab + rows)
    logits = (torch.randn(rows, vocab, generator=g, device="cuda") * 3 - 50).to(dtype)
    at = torch.randint(0, vocab, (rows, 3), generator=g, device="cuda")
    kinds = torch.tensor([math.nan, math.inf, -math.inf, -1000.0], device="cuda", dtype=dtype)
    logits.scatter_(1, at, kinds[torch.randint(0, 4, (rows, 3), generator=g, device="cuda")])
    open_ = torch.rand(rows, vocab, generator=g, device="cuda") < torch.tensor([0.5, 0.003, 1.0], device="cuda")[torch.arange(rows, device="cuda") % 3][:, None]
    open_[::4, at[0]] = True
    open_[1::7] = False
    words = -(-vocab // 32)
    bits = torch.nn.functional.pad(open_, (0, words * 32 - vocab)).view(rows, words, 32).long() << torch.arange(32, device="cuda")
    packed = bits.sum(-1)
    allowed = torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).int()
    heat = 0.02 + torch.rand(rows, generator=g, device="cuda")
    probs = torch.full((rows, vocab), -1.0, device="cuda")
    best = torch.empty(rows, dtype=torch.int32, device="cuda")
    logprob = torch.empty(rows, device="cuda")
    az.az_token_probs(logits, probs, best, logprob, allowed=allowed, temperature=heat)
    out = torch.empty_like(logits)
    az.az_adjust_logits(logits, out, allowed=allowed)
    assert torch.equal(out.nan_to_num(nan=7.0, posinf=8.0, neginf=9.0),
                       torch.where(open_, logits, -math.inf).nan_to_num(nan=7.0, posinf=8.0, neginf=9.0))
    line = torch.where(open_, logits.double(), -math.inf)
    nan = line.isnan().any(1)
    odd = nan | (line == math.inf).any(1)
    empty = ~odd & (line == -math.inf).all(1)
    assert odd.any() and empty.any() and (~odd & ~empty).any()
    assert (probs[~open_] == 0).all() and (probs[empty] == 0).all()
    assert probs[odd][open_[odd]].isnan().all() and logprob[odd].isnan().all()
    assert (best[empty] == -1).all() and (logprob[empty] == -math.inf).all()
    place = torch.arange(vocab, device="cuda")
    top = line.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).amax(1, keepdim=True)
    is_top = torch.where(nan[:, None], line.isnan(), line == top)
    lowest = torch.where(is_top & open_, place, vocab).amin(1)
    assert torch.equal(best.long()[~empty], lowest[~empty])
    fine = ~odd & ~empty
    x = (line - top) / heat.double()[:, None]
    want = x.exp() / x.exp().sum(1, keepdim=True)
    rel = (12 * 100 / heat.double()[:, None] + 5 * x.abs().clamp_max(1e4) + 120) * U
    assert ((probs.double() - want).abs() <= (rel + U) * want + smallest(F32))[fine].all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset,more", [(1, 0), (0, 1), (3, 5)])
def test_the_largest_vocabulary_at_any_alignment(az, dtype, offset, more):
    """Rows that take one chunk more than 16 CTAs of the usual share hold."""
    vocab, rows = 262144, 5
    flat = (torch.randn(offset + rows * (vocab + more), generator=gen(more + 7), device="cuda") * 4).to(dtype)
    logits = flat[offset:].view(rows, vocab + more)[:, :vocab]
    rules = make_rules(rows, vocab, 3, history=900, biases=60)
    check_logits(az, logits, rules, F32, vocab + more, offset)
    check_logits(az, logits, {"allowed": rules["allowed"]}, None, vocab + 8, 0)


def test_first_calls_from_several_threads_at_once():
    """The library's calls without the interpreter's lock, on a stream for each thread, from the process's first call on."""
    code = """
import ctypes, threading, torch
import paper_2609_37447_b200 as az
n, k, m, vocab = 9000, 512, 150, 9000
torch.manual_seed(1)
x, w = torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda")
p = lambda t: t.data_ptr()
def chain(stream, out):
    xq, xs, wq, ws, y, pr, best, lp = out
    s = stream.cuda_stream
    codes = [az._lib.az_quantise_blocks(p(w), 0, n, k, k, 128, p(wq), k, p(ws), 4, s), az._lib.az_quantise_blocks(p(x), 0, m, k, k, 1, p(xq), k, p(xs), 4, s),
             az._lib.az_block_matmul(p(xq), k, p(xs), 4, p(wq), k, p(ws), 4, None, m, n, k, p(y), 0, n, s),
             az._lib.az_token_probs(p(y), 0, m, vocab, n, None, p(pr), 0, n, p(best), p(lp), s)]
    assert codes == [0, 0, 0, 0], codes
def buffers():
    u8 = dict(dtype=torch.uint8, device="cuda")
    return [torch.empty(m, k, **u8), torch.empty(m, 4, device="cuda"), torch.empty(n, k, **u8), torch.empty(71, 4, device="cuda"),
            torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda"), torch.empty(m, dtype=torch.int32, device="cuda"), torch.empty(m, device="cuda")]
streams = [torch.cuda.Stream() for _ in range(6)]
outs = [[buffers() for _ in range(20)] for _ in streams]
torch.cuda.synchronize()
failed, gate = [], threading.Barrier(len(streams))
def work(i):
    try:
        gate.wait()
        for out in outs[i]:
            chain(streams[i], out)
    except BaseException as e:
        failed.append(e)
threads = [threading.Thread(target=work, args=(i,)) for i in range(len(streams))]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert not failed, failed
first = outs[0][0]
assert all(torch.equal(a, b) for o in outs for out in o for a, b in zip(first, out))
assert ((first[5].double().sum(1) - 1).abs() < 1e-4).all() and az.az_tokens_status() == 0
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), timeout=300)
