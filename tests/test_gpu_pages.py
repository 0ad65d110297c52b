"""The operators around the paged K/V store of eight bits, against their definitions in float64 (needs a B200)."""
import math

import numpy as np
import pytest
import torch

import paper_2608_22704_b200 as wnw
from pages_ref import E4M3, INT8, LOWEST, Store, attention, attention_bounds

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def starts_of(rows):
    return ints([0] + list(np.cumsum(rows)))


def randn(*shape, seed=0, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


# ---------------------------------------------------------------------------------------------------------------- rotate
def rotated(x, positions, plan, sign):
    """float64; x [tokens, heads, d], positions [axes][tokens]."""
    y = x.double().numpy().copy()
    n = plan.n_pairs
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if plan.neighbours else (i, i + n)
        t = sign * positions[plan.axis[i]].double().numpy() * plan.frequency[i]
        u, w = x[:, :, a].double().numpy(), x[:, :, b].double().numpy()
        y[:, :, a] = u * np.cos(t)[:, None] - w * np.sin(t)[:, None]
        y[:, :, b] = w * np.cos(t)[:, None] + u * np.sin(t)[:, None]
    return y


def check_rotated(got, x, positions, plan, sign):
    """Half a step of the type; below that the angle: reduced in 64 bits (2^-53 of it), as a fraction of a turn rounded to 32 (2^-26 of
    a turn at most: half a turn's last bit), sine and cosine to 2^-22, two products and a sum in fp32."""
    want = rotated(x, positions, plan, sign)
    n = plan.n_pairs
    size = np.abs(want)
    i = np.arange(n)
    a, b = (2 * i, 2 * i + 1) if plan.neighbours else (i, i + n)
    pair = np.abs(x.double().numpy()[:, :, a]) + np.abs(x.double().numpy()[:, :, b])
    far = positions.abs().double().max().item() * max(plan.frequency[:n]) * 2.0 ** -52
    err = np.zeros_like(want)
    err[:, :, a] = err[:, :, b] = pair * (2 * math.pi * 2.0 ** -26 + far + 2.0 ** -22 + 3 * 2.0 ** -24)
    err[:, :, 2 * n:] = 0.0
    tol = err + (size + err) * torch.finfo(got.dtype).eps / 2 + torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("d,pairs,sections,dealt,neighbours", [
    (128, 64, [16, 24, 24], False, False), (64, 32, [32], False, True), (128, 64, [24, 20, 20], True, False), (80, 20, [10, 10], False, False),
    (128, 48, [16, 16, 16], True, True), (6, 3, [1, 1, 1], False, False), (256, 128, [32, 32, 32, 32], True, False), (64, 1, [1], False, False)])
def test_rotate(dtype, d, pairs, sections, dealt, neighbours):
    plan = wnw.wnw_rotary_init(pairs, 1e6, sections, dealt, neighbours)
    for tokens, hq, hk in ((1, 16, 2), (37, 5, 5), (300, 8, 1)):
        q, k = randn(tokens, hq, d, seed=1, dtype=dtype), randn(tokens, hk, d, seed=2, dtype=dtype)
        pos = torch.randint(-50, 200000, (len(sections), tokens), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
        for inverse in (False, True):
            q_out, k_out = (torch.full_like(x, float("nan"), device=DEV) for x in (q, k))
            wnw.wnw_rotate(plan, pos.to(DEV), q.to(DEV), q_out, k.to(DEV), k_out, inverse=inverse)
            check_rotated(q_out, q, pos, plan, -1 if inverse else 1)
            check_rotated(k_out, k, pos, plan, -1 if inverse else 1)


def test_rotate_far_positions_and_odd_frequencies():
    plan = wnw.wnw_rotary_init(32, 1e4)
    for i in range(32):
        plan.frequency[i] *= 0.37 if i % 2 else -1.0
    x = randn(5, 2, 64, dtype=torch.float32)
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31, 10 ** 9, 1, 0]], dtype=torch.int32)
    out = torch.empty_like(x, device=DEV)
    wnw.wnw_rotate(plan, pos.to(DEV), x.to(DEV), out)
    check_rotated(out, x, pos, plan, 1)
    assert torch.equal(out[4].cpu(), x[4])


def test_rotate_in_place_strided_and_unaligned():
    plan = wnw.wnw_rotary_init(32, 1e4, [8, 12, 12])
    pos = torch.randint(0, 1000, (3, 50), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    wide = randn(50, 14, 80, seed=4)
    want = torch.empty(50, 8, 64, dtype=torch.bfloat16, device=DEV)
    wnw.wnw_rotate(plan, pos.to(DEV), wide[:, 2:10, :64].contiguous().to(DEV), want)
    for first in (0, 8, 3):                            # aligned as it comes, on 16 bytes, on 2
        host = torch.zeros(50, 14, 96, dtype=torch.bfloat16)
        host[:, :, first:first + 64] = wide[:, :, :64]
        dev = host.to(DEV)
        view = dev[:, 2:10, first:first + 64]
        wnw.wnw_rotate(plan, pos.to(DEV), view, view, dev[:, 10:13, first:first + 64], dev[:, 10:13, first:first + 64])
        assert torch.equal(view, want)
        check_rotated(dev[:, 10:13, first:first + 64], wide[:, 10:13, :64], pos, plan, 1)
        back = dev.cpu()
        back[:, 2:13, first:first + 64] = host[:, 2:13, first:first + 64]
        assert torch.equal(back, host)                 # nothing else was touched
    pos_wide = torch.zeros(3, 90, dtype=torch.int32, device=DEV)
    pos_wide[:, 20:70] = pos.to(DEV)
    out = torch.empty_like(want)
    wnw.wnw_rotate(plan, pos_wide[:, 20:70], wide[:, 2:10, :64].to(DEV), out)
    assert torch.equal(out, want)


def test_rotate_gradient():
    """The inverse is the transposed turn: against the formula's gradient by differences of a weighted sum, in fp32."""
    plan = wnw.wnw_rotary_init(16, 1e4, [8, 8])
    pos = torch.randint(0, 500, (2, 3), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    x, g = randn(3, 2, 40, seed=6, dtype=torch.float32), randn(3, 2, 40, seed=7, dtype=torch.float32)
    dx = torch.empty_like(x, device=DEV)
    wnw.wnw_rotate(plan, pos.to(DEV), g.to(DEV), dx, inverse=True)
    dx = dx.cpu().double().numpy()
    weigh = lambda z: float((rotated(z, pos, plan, 1) * g.double().numpy()).sum())  # noqa: E731
    for at in [(0, 0, 0), (1, 1, 15), (2, 0, 16), (2, 1, 31), (0, 1, 39)]:
        up, down = x.double().clone(), x.double().clone()
        up[at] += 0.5
        down[at] -= 0.5
        assert weigh(up) - weigh(down) == pytest.approx(dx[at], abs=1e-5)      # linear: a difference is the derivative


# --------------------------------------------------------------------------------------------------------- write and read
class Both:
    """A store on the GPU and its reference, one page table over both."""

    def __init__(self, n_pages, heads, T, d, fmt, n_seqs, width, seed=0, slack=0):
        self.ref = Store(n_pages, heads, T, d, fmt)
        rs = np.random.RandomState(seed)
        self.table = rs.permutation(n_pages)[:n_seqs * width].reshape(n_seqs, width)
        self.codes, self.scales = self.ref.to(DEV, slack)
        self.codes.view(torch.uint8).fill_(0x7f)            # what was there before must not matter
        self.scales.fill_(float("nan"))
        self.status = ints([0])
        self.pages = wnw.wnw_pages(self.codes, self.scales, self.status)
        self.table_dev = ints(self.table)
        self.lengths = [0] * n_seqs

    def write(self, k, v, rows, rotary=None, positions=None, max_rows=0, k_ref=None):
        starts = [0] + list(np.cumsum(rows))
        wnw.wnw_pages_write(self.pages, self.table_dev, ints(self.lengths), ints(starts), k, v, rotary=rotary, positions=positions, max_rows=max_rows)
        parts = lambda x: [x[a:b].double().cpu().numpy() for a, b in zip(starts, starts[1:])]  # noqa: E731
        self.ref.write(self.table, self.lengths, rows, parts(k if k_ref is None else k_ref), parts(v))
        self.lengths = [n + r for n, r in zip(self.lengths, rows)]

    def check(self):
        """Codes of every token held and the scales of its page, exactly."""
        codes, scales = self.codes.double().cpu().numpy(), self.scales.double().cpu().numpy()
        T = self.ref.T
        for s, n in enumerate(self.lengths):
            for i in range((n + T - 1) // T):
                page, rows = self.table[s, i], min(T, n - i * T)
                assert np.array_equal(scales[page], np.ldexp(1.0, self.ref.exps[page])), (s, i)
                assert np.array_equal(codes[page, :, :, :rows], self.ref.codes[page, :, :, :rows], equal_nan=True), (s, i)
        assert self.status.item() == 0


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("T,d,heads,dtype", [(16, 64, 3, torch.bfloat16), (64, 128, 2, torch.float16), (48, 128, 1, torch.bfloat16),
                                             (256, 128, 2, torch.bfloat16), (128, 64, 2, torch.float16)])
def test_write_grows_ragged_sequences(fmt, T, d, heads, dtype):
    """Prompts of all lengths, then pieces and single tokens, some larger than all before (scales rise), some of zeros."""
    n_seqs, width = 4, 1400 // T + 2
    b = Both(n_seqs * width + 3, heads, T, d, fmt, n_seqs, width, seed=T)
    for step, rows in enumerate([[1, 17, 0, 700], [1, 1, 1, 1], [0, T, T - 1, 5], [3, 1, 40, 0], [1, 1, 1, 1], [2 * T + 1, 1, 1, 33]]):
        scale = [1.0, 0.01, 30.0, 0.0, 2000.0, 1.0][step]
        k = randn(sum(rows), heads, d, seed=10 + step, dtype=dtype, scale=scale).to(DEV)
        v = randn(sum(rows), heads, d, seed=50 + step, dtype=dtype, scale=scale * 2.0 ** -8).to(DEV)
        b.write(k, v, rows, max_rows=(0, 1, max(rows), 1, 1, 7)[step])          # any value is safe
        b.check()


@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_write_of_every_bf16_magnitude(fmt):
    """Rows whose largest element is each of many bf16 numbers: the scale's borders, the smallest and the largest, infinities and NaN."""
    bits = np.concatenate([np.arange(0, 0x7f80, 47), np.arange(0x4300, 0x4400), [1, 2, 0x7f7f, 0x7f80, 0x7fc0, 0xff80, 0xffc0, 0x8000]]).astype(np.uint16)
    n = len(bits)
    x = torch.zeros(n, 1, 64, dtype=torch.int16)
    x[:, 0, 0] = torch.from_numpy(bits.view(np.int16))
    x[:, 0, 1:] = torch.randint(-2 ** 15, 2 ** 15, (n, 63), generator=torch.Generator().manual_seed(2)).to(torch.int16)
    x = x.view(torch.bfloat16)
    head = x[:, :, :1].abs().nan_to_num(nan=1.0, posinf=1.0)
    rest = torch.where(x[:, :, 1:].abs() <= head, x[:, :, 1:], torch.zeros_like(x[:, :, 1:]))        # (not-a-numbers go too)
    x = torch.cat([x[:, :, :1], rest], dim=2).to(DEV)
    b = Both(n, 1, 16, 64, fmt, n, 1)
    assert n <= 1024
    b.write(x, x, [1] * n)
    b.check()
    b.write(x.flip(0).contiguous(), x, [1] * n)          # a second token: scales rise or stay
    b.check()
    for dtype in (torch.bfloat16, torch.float16):
        k, v = (torch.empty(2 * n, 1, 64, dtype=dtype, device=DEV) for _ in range(2))
        wnw.wnw_pages_read(b.pages, b.table_dev, ints([0] * n), starts_of([2] * n), k, v)
        want = np.concatenate([b.ref.values(b.table[s], 2) for s in range(n)], axis=1)
        most = torch.finfo(dtype).max
        want = torch.tensor(np.clip(want, -most, most)).to(dtype)            # (exact in bf16; one rounding in fp16)
        assert torch.equal(torch.stack([k, v]).cpu().nan_to_num(nan=1.5), want.nan_to_num(nan=1.5))


@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_write_row_by_row_is_write_of_all_where_the_scale_is_settled(fmt):
    heads, d, T, n = 2, 128, 64, 150
    k, v = randn(n, heads, d, seed=1).to(DEV), randn(n, heads, d, seed=2).to(DEV)
    for x in (k, v):                                       # the first row of each page has its largest element
        for t in range(0, n, T):
            x[t] = 7.0
    one, all_ = (Both(4, heads, T, d, fmt, 1, 4) for _ in range(2))
    all_.write(k, v, [n])
    for t in range(n):
        one.write(k[t:t + 1], v[t:t + 1], [1])
    one.check()
    for i in range(3):
        rows = min(T, n - i * T)
        p, q = one.table[0, i], all_.table[0, i]
        assert torch.equal(one.codes.view(torch.uint8)[p, :, :, :rows], all_.codes.view(torch.uint8)[q, :, :, :rows])


@pytest.mark.parametrize("neighbours,pairs", [(False, 64), (True, 64), (False, 24), (True, 16)])
@pytest.mark.parametrize("T,dtype", [(64, torch.bfloat16), (256, torch.float16), (16, torch.bfloat16), (128, torch.bfloat16)])
def test_write_turns_keys_as_rotate_does(neighbours, pairs, T, dtype):
    heads, d, rows = 3, 128, [1, 100, 0, 300]
    plan = wnw.wnw_rotary_init(pairs, 1e4, [pairs // 2, pairs - pairs // 2], neighbours=neighbours)
    pos = torch.randint(0, 10 ** 6, (2, sum(rows)), generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(DEV)
    k, v = randn(sum(rows), heads, d, seed=3, dtype=dtype).to(DEV), randn(sum(rows), heads, d, seed=4, dtype=dtype).to(DEV)
    turned = torch.empty_like(k)
    wnw.wnw_rotate(plan, pos, k, turned)
    width = 310 // T + 1
    b = Both(4 * width, heads, T, d, INT8, 4, width)
    b.write(k, v, rows, rotary=plan, positions=pos, k_ref=turned)
    b.check()
    b.write(k[:4], v[:4], [1] * 4, rotary=plan, positions=pos[:, :4], k_ref=turned[:4])
    b.check()


@pytest.mark.parametrize("fmt,dtype", [(E4M3, torch.bfloat16), (INT8, torch.bfloat16), (E4M3, torch.float16), (INT8, torch.float16)])
def test_read_back(fmt, dtype):
    heads, d, T = 3, 128, 48
    b = Both(20, heads, T, d, fmt, 3, 6, slack=64)
    rows = [1, 130, 288]
    b.write(randn(sum(rows), heads, d, seed=1, dtype=dtype, scale=9.0).to(DEV), randn(sum(rows), heads, d, seed=2, dtype=dtype).to(DEV), rows)
    b.check()
    for first, count in (([0, 0, 0], rows), ([0, 47, 49], [1, 2, 100]), ([0, 129, 287], [0, 1, 1])):
        n = sum(count)
        wide = torch.full((n + 2, 2, heads + 1, d), 5.0, dtype=dtype, device=DEV)      # slices of a wider tensor, rows behind the last
        k, v = wide[:, 0, :heads], wide[:, 1, :heads]
        wnw.wnw_pages_read(b.pages, b.table_dev, ints(first), starts_of(count), k, v, max_rows=max(count))
        at = 0
        for s in range(3):
            want = b.ref.values(b.table[s], first[s] + count[s])[:, first[s]:]
            for x, w in ((k, 0), (v, 1)):
                assert np.array_equal(x[at:at + count[s]].double().cpu().numpy(), want[w])
            at += count[s]
        assert (wide[n:] == 5.0).all() and (wide[:, :, heads] == 5.0).all()
    assert b.status.item() == 0


def test_read_of_what_fp16_cannot_hold():
    b = Both(1, 1, 16, 64, E4M3, 1, 1)
    x = torch.full((1, 1, 64), 65504.0, dtype=torch.float16, device=DEV)       # stored as 65536
    x[0, 0, 1] = -65504.0
    b.write(x, x, [1])
    b.check()
    k, v = torch.empty_like(x), torch.empty_like(x)
    wnw.wnw_pages_read(b.pages, b.table_dev, ints([0]), ints([0, 1]), k, v)
    assert torch.equal(k, x) and torch.equal(v, x)


def test_pages_beyond_32_bits():
    """Pages 3 GB apart."""
    heads, T, d = 1, 16, 64
    size, apart = 2 * T * d, 3 << 30
    raw = torch.empty(2 * apart + size, dtype=torch.uint8, device=DEV)
    codes = raw.view(torch.int8).as_strided((3, heads, 2, T, d), (apart, size, T * d, d, 1))
    scales = torch.zeros(3, heads, 2, device=DEV)
    pages = wnw.wnw_pages(codes, scales)
    table, rows = ints([[2, 0, 1]]), 40
    k, v = randn(rows, 1, d, seed=1).to(DEV), randn(rows, 1, d, seed=2).to(DEV)
    wnw.wnw_pages_write(pages, table, ints([0]), ints([0, rows]), k, v)
    ref = Store(3, heads, T, d, INT8)
    ref.write([[2, 0, 1]], [0], [rows], [k.double().cpu().numpy()], [v.double().cpu().numpy()])
    want = ref.values([2, 0, 1], rows)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    wnw.wnw_pages_read(pages, table, ints([0]), ints([0, rows]), k2, v2)
    assert np.array_equal(k2.double().cpu().numpy(), want[0]) and np.array_equal(v2.double().cpu().numpy(), want[1])
    q = randn(1, 2, d, seed=3).to(DEV)
    out, lse = attend(pages, table, [rows], [1], q)
    check_attention(out, lse, q, [want], [rows], [1], True)


# ---------------------------------------------------------------------------------------------------------------- attend
def workspace_for(pages, hq):
    return torch.full((wnw.wnw_pages_attend_workspace(pages, hq),), 0xff, dtype=torch.uint8, device=DEV)     # NaN as floats


def attend(pages, table, lengths, rows, q, causal=True, scale=0.0, max_rows=0, extra=0):
    out = torch.full((q.shape[0], q.shape[1], q.shape[2]), 7.0, dtype=q.dtype, device=DEV)
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device=DEV)
    wnw.wnw_pages_attend(pages, table, ints(lengths), starts_of(rows), q, out, workspace_for(pages, q.shape[1]), lse=lse, causal=causal,
                         softmax_scale=scale, max_rows=max_rows)
    return out, lse


def check_attention(out, lse, q, values, lengths, rows, causal, scale=0.0, T=256):
    """values: per sequence [2][tokens, heads, d] as stored."""
    d = q.shape[2]
    scale = scale or 1.0 / math.sqrt(d)
    at = 0
    for s, (n, r) in enumerate(zip(lengths, rows)):
        end = [n - r + i + 1 if causal else n for i in range(r)]
        want, want_lse, spread, reach = attention(q[at:at + r].double().cpu().numpy(), values[s][0], values[s][1], end, scale, T)
        tol, tol_lse = attention_bounds(want, want_lse, spread, reach, q.dtype, d)
        got, got_lse = out[at:at + r].double().cpu().numpy(), lse[at:at + r].double().cpu().numpy()
        bad = np.isnan(want)
        assert np.array_equal(np.isnan(got), bad), s
        assert (np.abs(got - want)[~bad] <= tol[~bad]).all(), (s, np.abs(got - want)[~bad].max(), (np.abs(got - want) / tol)[~bad].max())
        gone = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse), gone) and (got[gone] == 0).all()
        fine = np.isfinite(want_lse)
        assert (np.abs(got_lse[fine] - want_lse[fine]) <= tol_lse[fine]).all(), (s, np.abs(got_lse[fine] - want_lse[fine]).max())
        at += r
    assert (out[at:] == 7.0).all() and (lse[at:] == 7.0).all()              # rows behind the last sequence's


def filled(fmt, heads, T, d, lengths, seed=0, dtype=torch.bfloat16, k_scale=1.0, v_scale=1.0, slack=0):
    width = max(1, max((n + T - 1) // T for n in lengths))
    b = Both(len(lengths) * width + 2, heads, T, d, fmt, len(lengths), width, seed=seed, slack=slack)
    if sum(lengths):
        b.write(randn(sum(lengths), heads, d, seed=seed + 1, dtype=dtype, scale=k_scale).to(DEV),
                randn(sum(lengths), heads, d, seed=seed + 2, dtype=dtype, scale=v_scale).to(DEV), lengths)
    return b


def values_of(b, lengths):
    return [b.ref.values(b.table[s], n) for s, n in enumerate(lengths)]


LENGTHS = [0, 1, 15, 16, 17, 300, 1291]


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("hq,heads,d,T,dtype", [(8, 4, 64, 32, torch.bfloat16), (32, 8, 128, 64, torch.bfloat16), (16, 2, 128, 16, torch.float16),
                                                (5, 5, 64, 48, torch.float16), (28, 4, 128, 128, torch.bfloat16), (20, 2, 64, 64, torch.bfloat16),
                                                (16, 1, 128, 256, torch.float16), (9, 3, 128, 64, torch.float16)])
def test_attend_one_token(fmt, hq, heads, d, T, dtype):
    b = filled(fmt, heads, T, d, LENGTHS, seed=hq, dtype=dtype)
    q = randn(len(LENGTHS) + 2, hq, d, seed=9, dtype=dtype, scale=2.0).to(DEV)
    for causal in (True, False):
        out, lse = attend(b.pages, b.table_dev, LENGTHS, [1] * len(LENGTHS), q, causal=causal, max_rows=1)
        check_attention(out, lse, q, values_of(b, LENGTHS), LENGTHS, [1] * len(LENGTHS), causal)
    assert b.status.item() == 0


ROWS = [2, 3, 0, 20, 17, 4, 33]          # more rows than tokens: the first see nothing


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("hq,heads,d,T", [(8, 4, 64, 32), (16, 2, 128, 64), (5, 5, 128, 16), (20, 2, 64, 48), (28, 4, 128, 64), (16, 1, 128, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_several_rows(fmt, hq, heads, d, T, causal):
    b = filled(fmt, heads, T, d, LENGTHS, seed=hq)
    q = randn(sum(ROWS) + 3, hq, d, seed=9, scale=2.0).to(DEV)
    for max_rows in (1, 4, 33, 0):
        out, lse = attend(b.pages, b.table_dev, LENGTHS, ROWS, q, causal=causal, max_rows=max_rows)
        check_attention(out, lse, q, values_of(b, LENGTHS), LENGTHS, ROWS, causal)


@pytest.mark.parametrize("fmt,heads,d,lengths,rows", [(E4M3, 8, 128, [4000], [130]), (INT8, 4, 64, [3000, 1, 2500], [70, 1, 200]), (E4M3, 4, 64, [1500, 1400, 0], [300, 65, 3]),
                                                      (INT8, 6, 128, [2600], [65])])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_prompts(fmt, heads, d, lengths, rows, causal):
    """Many tiles of tokens to a CTA, items of one and of two row tiles beside one another, items that several CTAs share."""
    b = filled(fmt, heads, 64, d, lengths, seed=heads)
    q = randn(sum(rows) + 1, 4 * heads, d, seed=9, scale=2.0).to(DEV)
    out, lse = attend(b.pages, b.table_dev, lengths, rows, q, causal=causal)
    check_attention(out, lse, q, values_of(b, lengths), lengths, rows, causal)
    assert b.status.item() == 0


@pytest.mark.parametrize("fmt,hq,heads,d", [(E4M3, 32, 8, 128), (INT8, 16, 2, 128), (E4M3, 8, 4, 64)])
def test_attend_long_and_many(fmt, hq, heads, d):
    """One head spread over every CTA; and more heads than a CTA prepares at a time."""
    b = filled(fmt, 1, 64, d, [20011], seed=3)
    q = randn(1, hq // heads, d, seed=9, scale=2.0).to(DEV)
    out, lse = attend(b.pages, b.table_dev, [20011], [1], q, max_rows=1)
    check_attention(out, lse, q, values_of(b, [20011]), [20011], [1], True)
    lengths = [int(x) for x in np.random.RandomState(1).randint(0, 60, 700)]
    rows = [int(x) for x in np.random.RandomState(2).randint(0, 3, 700)]
    b = filled(fmt, heads, 16, d, lengths, seed=4)
    q = randn(sum(rows) + 1, hq, d, seed=9, scale=2.0).to(DEV)
    out, lse = attend(b.pages, b.table_dev, lengths, rows, q)
    check_attention(out, lse, q, values_of(b, lengths), lengths, rows, True)


@pytest.mark.parametrize("rows", [1, 30])
@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_attend_scales_far_apart(fmt, rows):
    """Pages whose values differ by 2^60, in both orders, and weights that the small ones carry; then pages of zeros among them."""
    heads, T, d, n = 2, 16, 64, 640
    for order in (1, -1, 0):
        b = Both(42, heads, T, d, fmt, 1, 40)
        k, v = randn(n, heads, d, seed=1).to(DEV), randn(n, heads, d, seed=2).to(DEV)
        power = torch.arange(n // T, device=DEV).repeat_interleave(T).float()
        power = (power if order > 0 else power.flip(0)) * 1.5 - 30
        if order:
            v = (v.float() * torch.exp2(power)[:, None, None]).to(torch.bfloat16)
        else:
            v[64:n - 64].view(-1, T, heads, d)[::2] = 0.0
            v[n // 2:n - 16] = 0.0
        b.write(k, v, [n])
        q = randn(rows, 4, d, seed=3, scale=30.0).to(DEV)             # one key has nearly all the weight
        for scale in (0.0, 3.0, 1e-3):
            out, lse = attend(b.pages, b.table_dev, [n], [rows], q, scale=scale)
            check_attention(out, lse, q, values_of(b, [n]), [n], [rows], True, scale, T)


@pytest.mark.parametrize("dtype,size,scale", [(torch.bfloat16, 1e25, 1e-26), (torch.bfloat16, 1e-25, 1e24), (torch.float16, 6e4, 1e-5), (torch.bfloat16, 0.0, 0.0)])
def test_attend_queries_of_any_size(dtype, size, scale):
    b = filled(E4M3, 2, 32, 64, [500])
    q = randn(1, 4, 64, seed=3).clamp(-1, 1).mul(size).to(dtype).to(DEV)
    out, lse = attend(b.pages, b.table_dev, [500], [1], q, scale=scale)
    check_attention(out, lse, q, values_of(b, [500]), [500], [1], True, scale)


def test_attend_not_a_numbers_reach_only_those_who_see_them():
    heads, T, d, n, rows = 2, 32, 128, 150, 30
    for at_k, at_v in ((140, None), (None, 140), (None, 128), (149, 3)):
        b = Both(8, heads, T, d, E4M3, 1, 6)
        k, v = randn(n, heads, d, seed=1).to(DEV), randn(n, heads, d, seed=2).to(DEV)
        if at_k is not None:
            k[at_k, 1, 5] = float("nan")
        if at_v is not None:
            v[at_v, 0, 77] = float("nan")
        b.write(k, v, [n])
        b.check()
        q = randn(rows, 8, d, seed=3).to(DEV)
        for causal in (True, False):
            out, lse = attend(b.pages, b.table_dev, [n], [rows], q, causal=causal)
            check_attention(out, lse, q, values_of(b, [n]), [n], [rows], causal)
    q[3, 2, 9] = float("nan")
    q[4, 6, 0] = float("inf")
    out, lse = attend(b.pages, b.table_dev, [100], [rows], q)
    bad = torch.zeros(rows, 8, dtype=torch.bool, device=DEV)
    bad[3, 2] = bad[4, 6] = True
    bad[:, :4] |= (v[3:4, 0].isnan().any() & (torch.arange(rows, device=DEV) >= 0))[:, None]
    assert torch.equal(out.isnan().any(-1) | lse.isnan(), bad)


def test_bad_pages_and_lengths_are_left_out_and_reported():
    heads, T, d = 2, 16, 64
    lengths = [50, 70]
    b = filled(INT8, heads, T, d, lengths)
    values = values_of(b, lengths)
    q = randn(2, 4, d, seed=3).to(DEV)
    for wrong in (-1, b.pages.n_pages, 2 ** 31 - 1, -2 ** 31):
        b.status.zero_()
        table = b.table_dev.clone()
        table[1, 1] = wrong
        out, lse = attend(b.pages, table, lengths, [1, 1], q, max_rows=1)
        assert b.status.item() == wnw.WNW_PAGES_BAD_PAGE
        kept = np.concatenate([values[1][:, :16], values[1][:, 32:]], axis=1)
        check_attention(out, lse, q, [values[0], kept], [50, 54], [1, 1], False)
        b.status.zero_()
        k, v = torch.ones(120, heads, d, device=DEV, dtype=torch.bfloat16), torch.ones(120, heads, d, device=DEV, dtype=torch.bfloat16)
        wnw.wnw_pages_read(b.pages, table, ints([0, 0]), ints([0, 50, 120]), k, v)
        assert b.status.item() == wnw.WNW_PAGES_BAD_PAGE and (k[66:82] == 0).all() and (v[66:82] == 0).all() and (k[50:66] != 0).any()
        before = b.codes.clone()
        b.status.zero_()
        wnw.wnw_pages_write(b.pages, table, ints([50, 16]), ints([0, 0, 16]), k[:16], v[:16])
        assert b.status.item() == wnw.WNW_PAGES_BAD_PAGE and torch.equal(before, b.codes)
    width = b.table.shape[1]
    for bad in ([50, -1], [50, width * T + 1], [2 ** 31 - 1, 70]):
        b.status.zero_()
        out, lse = attend(b.pages, b.table_dev, bad, [1, 1], q, causal=False, max_rows=1)
        assert b.status.item() == wnw.WNW_PAGES_BAD_LENGTH
        if bad[1] < 0:
            assert (out[1] == 0).all() and lse[1].isneginf().all()
        good = 1 if bad[0] > 1000 else 0
        check_attention(out[good:good + 1], lse[good:good + 1], q[good:good + 1], [values[good]], [lengths[good]], [1], False)
    for starts in ([0, 1, 3], [0, -5, 2], [0, 2, 1], [2 ** 31 - 1, 0, 1]):            # rows that are not there
        b.status.zero_()
        out = torch.zeros_like(q)
        wnw.wnw_pages_attend(b.pages, b.table_dev, ints(lengths), ints(starts), q, out, workspace_for(b.pages, 4))
        assert b.status.item() == wnw.WNW_PAGES_BAD_LENGTH
        b.status.zero_()
        before = b.codes.clone()
        wnw.wnw_pages_write(b.pages, b.table_dev, ints([50, 70]), ints([3, 1, 1]), k[:2], v[:2])
        assert b.status.item() == wnw.WNW_PAGES_BAD_LENGTH and torch.equal(before, b.codes)


def test_strides_of_queries_and_outputs():
    b = filled(E4M3, 2, 64, 128, [333, 80], slack=4096)
    wide = randn(7, 12, 128, seed=3).to(DEV)
    q = wide[:5, 4:12]
    room = torch.full((5, 20, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    out = room[:, 10:18]
    wnw.wnw_pages_attend(b.pages, b.table_dev, ints([333, 80]), ints([0, 3, 5]), q, out, workspace_for(b.pages, 8))
    want, lse = attend(b.pages, b.table_dev, [333, 80], [3, 2], q.contiguous())
    check_attention(want, lse, q.contiguous(), values_of(b, [333, 80]), [333, 80], [3, 2], True)
    assert torch.equal(out, want) and (room[:, :10] == 7).all() and (room[:, 18:] == 7).all()
    table = torch.zeros(2, b.table_dev.shape[1] + 5, dtype=torch.int32, device=DEV)         # a wider table, as a pool keeps it
    table[:, :b.table_dev.shape[1]] = b.table_dev
    again, _ = attend(b.pages, table[:, :b.table_dev.shape[1]], [333, 80], [3, 2], q.contiguous())
    assert torch.equal(again, want)


@pytest.mark.parametrize("lengths,rows", [([5000, 123, 777], 1), ([40000], 1), ([5000, 123, 777], 70)])
def test_attend_gives_the_same_bits_again(lengths, rows):
    b = filled(E4M3, 4, 64, 128, lengths)
    q = randn(rows * len(lengths), 16, 128, seed=3, scale=2.0).to(DEV)
    first = attend(b.pages, b.table_dev, lengths, [rows] * len(lengths), q)
    for _ in range(5):
        again = attend(b.pages, b.table_dev, lengths, [rows] * len(lengths), q)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_attend_in_clusters_and_on_the_line():
    """Short sequences under a table of any width: what the call may have to read decides how it is cut, not what it gives."""
    lengths = [300, 17, 0, 1]
    b = filled(INT8, 2, 64, 128, lengths)
    for rows, hq in ((1, 8), (3, 10)):
        q = randn(4 * rows, hq, 128, seed=3, scale=2.0).to(DEV)
        for width in (b.table_dev.shape[1], 40, 4000):
            table = torch.full((4, width), 10 ** 9, dtype=torch.int32, device=DEV)         # never looked at
            table[:, :b.table_dev.shape[1]] = b.table_dev
            out, lse = attend(b.pages, table, lengths, [rows] * 4, q, max_rows=rows)
            check_attention(out, lse, q, values_of(b, lengths), lengths, [rows] * 4, True)
    assert b.status.item() == 0


def test_a_captured_step_replayed_while_sequences_grow():
    """Rotate, write and attend captured once, replayed with lengths that move on, beside another graph with a workspace of its own."""
    heads, hq, T, d, n_seqs = 2, 8, 16, 64, 3
    plan = wnw.wnw_rotary_init(32, 1e4, [8, 12, 12])
    b = Both(30, heads, T, d, E4M3, n_seqs, 8)
    prompt = [20, 1, 47]
    b.write(randn(sum(prompt), heads, d, seed=1).to(DEV), randn(sum(prompt), heads, d, seed=2).to(DEV), prompt)
    steps = 20
    q, k, v = (randn(steps, n_seqs, h, d, seed=s).to(DEV) for h, s in ((hq, 3), (heads, 4), (heads, 5)))
    pos = torch.randint(0, 1000, (steps, 3, n_seqs), generator=torch.Generator().manual_seed(6), dtype=torch.int32).to(DEV)
    qs, ks, vs, ps = (x[0].clone() for x in (q, k, v, pos))
    lengths, after = ints(prompt), ints(prompt)
    starts, q_turned, out = starts_of([1] * n_seqs), torch.empty_like(qs), torch.empty_like(qs)
    lse, ws = torch.empty(n_seqs, hq, device=DEV), workspace_for(b.pages, hq)

    def step():
        torch.add(lengths, 1, out=after)
        wnw.wnw_rotate(plan, ps, qs, q_turned)
        wnw.wnw_pages_write(b.pages, b.table_dev, lengths, starts, ks, vs, rotary=plan, positions=ps, max_rows=1)
        wnw.wnw_pages_attend(b.pages, b.table_dev, after, starts, q_turned, out, ws, lse=lse, max_rows=1)
        lengths.copy_(after)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()                                              # a first run outside the capture
        side.synchronize()
        lengths.copy_(ints(prompt))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for t in range(steps):
        turned_k = torch.empty_like(k[t])
        wnw.wnw_rotate(plan, pos[t], k[t], turned_k)
        for dst, src in ((qs, q[t]), (ks, k[t]), (vs, v[t]), (ps, pos[t])):
            dst.copy_(src)
        # (the first run wrote token 0 already: the same codes again)
        b.ref.write(b.table, b.lengths, [1] * n_seqs, [x[None].double().cpu().numpy() for x in turned_k], [x[None].double().cpu().numpy() for x in v[t]])
        graph.replay()
        torch.cuda.synchronize()
        b.lengths = [n + 1 for n in b.lengths]
        b.check()
        check_attention(out, lse, q_turned, values_of(b, b.lengths), b.lengths, [1] * n_seqs, True)
    assert lengths.tolist() == b.lengths


def test_two_streams_with_a_workspace_each():
    lengths = [9000, 8000]
    b = filled(E4M3, 4, 64, 128, lengths)
    q = [randn(2, 16, 128, seed=s, scale=2.0).to(DEV) for s in (3, 4)]
    want = [attend(b.pages, b.table_dev, lengths, [1, 1], x)[0] for x in q]
    streams, ws = [torch.cuda.Stream(), torch.cuda.Stream()], [workspace_for(b.pages, 16) for _ in range(2)]
    out = [[torch.empty_like(x) for _ in range(10)] for x in q]
    n, starts = ints(lengths), ints([0, 1, 2])
    torch.cuda.synchronize()
    for i in range(10):
        for j in range(2):
            wnw.wnw_pages_attend(b.pages, b.table_dev, n, starts, q[j], out[j][i], ws[j], stream=streams[j])
    torch.cuda.synchronize()
    for j in range(2):
        for x in out[j]:
            assert torch.equal(x, want[j])


def test_arguments_that_the_binding_refuses():
    b = filled(E4M3, 2, 16, 64, [40])
    q = randn(1, 4, 64).to(DEV)
    out, ws = torch.empty_like(q), workspace_for(b.pages, 4)
    args = lambda **kw: {**dict(pages=b.pages, page_table=b.table_dev, lengths=ints([40]), row_starts=ints([0, 1]), q=q, out=out, workspace=ws), **kw}  # noqa: E731
    wnw.wnw_pages_attend(**args())
    for kw in (dict(page_table=b.table_dev.long()), dict(lengths=ints([40, 2])), dict(row_starts=ints([0])), dict(q=q.float()), dict(out=out.half()),
               dict(q=q[:, :, :32]), dict(q=q.cpu()), dict(workspace=ws[:100]), dict(workspace=ws[16:]), dict(lse=torch.zeros(1, 4)),
               dict(lse=torch.zeros(1, 5, device=DEV)), dict(lengths=ints([40]).cpu()), dict(out=torch.empty(1, 8, 64, device=DEV, dtype=q.dtype))):
        with pytest.raises(wnw.WnwError):
            wnw.wnw_pages_attend(**args(**kw))
    for codes, scales in ((b.codes.float(), b.scales), (b.codes, b.scales.double()), (b.codes[:, :1], b.scales), (b.codes.cpu(), b.scales),
                          (b.codes.transpose(3, 4), b.scales), (b.codes, b.scales.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(wnw.WnwError):
            wnw.wnw_pages(codes, scales)
    plan = wnw.wnw_rotary_init(32, 1e4, [16, 16])
    for kw in (dict(positions=ints([3])), dict(positions=ints([[3], [4]]).long()), dict(positions=ints([[3], [4]]), k=q), dict(q_out=out[:, :2])):
        with pytest.raises(wnw.WnwError):
            wnw.wnw_rotate(**{**dict(rotary=plan, positions=ints([[3], [4]]), q=q, q_out=out), **kw})
    k = randn(2, 2, 64).to(DEV)
    for kw in (dict(k=k[:, :1]), dict(v=k.half()), dict(rotary=plan), dict(positions=ints([[3, 4], [4, 5]])), dict(rotary=plan, positions=ints([3, 4]))):
        with pytest.raises(wnw.WnwError):
            wnw.wnw_pages_write(**{**dict(pages=b.pages, page_table=b.table_dev, lengths=ints([0]), row_starts=ints([0, 2]), k=k, v=k), **kw})


# ------------------------------------------------------------------------------------------------------- with the framework
@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_pages_hand_a_prompt_over_to_a_cache(fmt):
    """A prompt kept in eight-bit pages, turned as it was written, comes back as the prefill of a cache: attention over the pages, over a
    caller-owned buffer and through the cache agree."""
    heads, hq, T, d, n = 4, 16, 64, 128, 777
    plan = wnw.wnw_rotary_init(64, 1e6, [16, 24, 24])
    pos = torch.arange(n, dtype=torch.int32, device=DEV).repeat(3, 1)
    k, v = randn(n, heads, d, seed=1).to(DEV), randn(n, heads, d, seed=2).to(DEV)
    turned = torch.empty_like(k)
    wnw.wnw_rotate(plan, pos, k, turned)
    b = Both(16, heads, T, d, fmt, 1, 13)
    b.write(k[:700], v[:700], [700], rotary=plan, positions=pos[:, :700], k_ref=turned[:700])
    b.write(k[700:], v[700:], [77], rotary=plan, positions=pos[:, 700:], k_ref=turned[700:])
    b.check()
    q = randn(1, hq, d, seed=3, scale=2.0).to(DEV)
    q_turned = torch.empty_like(q)
    wnw.wnw_rotate(plan, ints([[n - 1]] * 3), q, q_turned)
    out, lse = attend(b.pages, b.table_dev, [n], [1], q_turned)
    values = values_of(b, [n])
    check_attention(out, lse, q_turned, values, [n], [1], True)

    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    wnw.wnw_pages_read(b.pages, b.table_dev, ints([0]), ints([0, n]), k2, v2)
    kv = torch.zeros(heads, 2, 784, d, dtype=torch.bfloat16, device=DEV)
    kv[:, 0, :n], kv[:, 1, :n] = k2.transpose(0, 1), v2.transpose(0, 1)
    static = torch.empty(hq, d, dtype=torch.bfloat16, device=DEV)
    wnw.wnw_attend_static(kv, n, q_turned[0], static)
    cache = wnw.wnw_create(1, hq, heads, d, 1, n, 16, 16, 1.0, np.zeros(heads, np.uint8), mode=wnw.WNW_MODE_FULL)
    try:
        wnw.wnw_place_prefill(cache, 0, 0, k2, v2, 0, n)
        full = torch.empty(1, hq, d, dtype=torch.bfloat16, device=DEV)
        wnw.wnw_step_begin(cache, [0])
        wnw.wnw_decode_layer_full(cache, 0, q_turned, None, None, full)
        wnw.wnw_step_end(cache)
        wnw.wnw_sync(cache)
    finally:
        wnw.wnw_destroy(cache)
    for other in (static, full[0]):            # bf16 weights and outputs of O(1)
        assert (other.float() - out[0].float()).abs().max() <= 2e-2
