"""The embedding operators (typed lookup with scaling and dropout, its gradient by sorted slots, the step of the touched
rows) against their formulas in 64 bits.

Tolerances count roundings.  u = 2^-24 is half a step of a 32-bit float, h half a step of the type of the result.
  lookup    f is rounded once, the product once, the result once:                  |error| <= (2 u + h) |result|, and h of the
            type's smallest step where the result is subnormal
  gradient  a sum of k terms in any order has at most k - 1 roundings of partial sums, each at most the sum of the terms'
            absolute values S; f, the product with it and the result are rounded:  |error| <= (k + 2) u S + h |result|
  step      with |error of G| <= e_G as above without h:  SGD  |error| <= lr e_G + 4 u (|w| + |lr G|) + h |result|.
            Adagrad: the mean of G^2 has an error of 2 e_G |G| + e_G^2 + (dim + 4) u G^2 per element, the state another
            rounding: e_s in all.  The change lr G / (sqrt(state) + eps) grows with |G| and falls, ever more slowly, with the
            state: with a state off by e_s it is off by no more than at low = max(state - e_s, what the state was before), so by
            lr (|G| + e_G) / (sqrt(low) + eps) - lr |G| / (sqrt(state) + eps) at most; its own 6 roundings are 6 u of its largest.
(second-order terms are covered by a factor of 1.01)"""
import math

import numpy as np
import pytest
import torch

import embed_reference as ref
from paper_2602_17050_amd import binding as mp
from paper_2602_17050_amd import workloads as wl
from gpu_common import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SMALLEST = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}


def half_step(t):
    return torch.finfo(t).eps / 2


def f64(t):
    return t.double().cpu().numpy()


def seed_tensor(seed):
    return torch.tensor([seed - (1 << 64) if seed >= 1 << 63 else seed], dtype=torch.int64, device="cuda")


def close(got, want, error, what):
    off = np.abs(got - want)
    with np.errstate(invalid="ignore"):
        bad = ~((off <= error) | (np.isnan(got) & np.isnan(want)) | (got == want))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5])


@pytest.fixture(scope="module")
def handle():
    h = mp.mpzch_embed_create()
    yield h
    mp.mpzch_embed_destroy(h)


def adagrad_errors(total, e_g, state_before, state, lr, eps):
    """(error of the state, of the change) as derived above, for the rows named"""
    dim = total.shape[1]
    e_state = (2 * e_g * np.abs(total) + e_g ** 2 + (dim + 4) * U * total ** 2).mean(1) + 2 * U * state
    low = np.maximum(state - 1.01 * e_state, state_before * (1 - 2 * U))
    most = lr * (np.abs(total) + e_g) / (np.sqrt(low) + eps)[:, None]
    return e_state, most - lr * np.abs(total) / (np.sqrt(state) + eps)[:, None] + 6 * U * most


def draw_slots(rng, n, num_rows, kind):
    if kind == "same":
        return np.full(n, int(rng.integers(num_rows)), dtype=np.int64)
    if kind == "distinct":
        return rng.permutation(max(n, num_rows))[:n].astype(np.int64)
    if kind == "padding":
        return np.full(n, -1, dtype=np.int64)
    if kind == "beyond":                                       # slots beyond the rows: row = slot mod rows
        return rng.integers(0, 1 << 62, size=n)
    s = (wl.zipf_ranks(rng, n, 1.1, num_rows) - 1) * 7919 % num_rows
    s[rng.random(n) < 0.1] = -(1 + int(rng.integers(1 << 40)))
    return s.astype(np.int64)


def tensor2d(rng, n, dim, dtype, layout="dense", scale=1.0):
    """n x dim values; "wide": columns of a wider tensor that start at an odd element, "padded": rows further apart"""
    x = torch.from_numpy(rng.standard_normal((n, dim)) * scale).to(dtype)
    if layout == "dense":
        return x.cuda()
    extra = 3 if layout == "wide" else 8
    big = torch.zeros(n, dim + extra, dtype=dtype, device="cuda")
    view = big[:, 1:1 + dim] if layout == "wide" else big[:, :dim]
    view.copy_(x)
    return view


# ------------------------------------------------------------------------------------------------ lookup
EMBED = [(1, 1, 1, F32, F32), (1, 7, 16, BF16, BF16), (2, 1, 3, F32, F16), (63, 10, 4, F16, F32), (64, 1000, 64, BF16, BF16),
         (257, 999, 50, F32, BF16), (1000, 50, 333, F16, F16), (333, 4099, 128, BF16, F32), (7, 100, 4096, BF16, BF16),
         (5, 3, 5001, F32, F32), (20_011, 50_021, 48, F32, BF16), (100_003, 1000, 8, F16, BF16), (4097, 300, 1, BF16, F32),
         (3, 2, 1 << 20, BF16, F32)]


@pytest.mark.parametrize("n,num_rows,dim,table,out_type", EMBED)
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_embed(n, num_rows, dim, table, out_type, p):
    rng = np.random.Generator(np.random.Philox(key=n * 1000 + dim))
    for layout in ("dense", "wide", "padded"):
        rows = tensor2d(rng, num_rows, dim, table, layout)
        out = tensor2d(rng, n, dim, out_type, layout)
        behind = out.untyped_storage().nbytes()
        slots_np = draw_slots(rng, n, num_rows, "zipf" if layout == "dense" else "beyond")
        seed, scale = int(rng.integers(1 << 63)) * 2 + 1, float(np.float32(math.sqrt(dim)))
        say("embed", n, num_rows, dim, table, out_type, p, layout, behind)
        mp.mpzch_embed(torch.from_numpy(slots_np).cuda(), rows, out, scale=scale, drop_p=p, seed=seed_tensor(seed))
        want = ref.embed(slots_np, f64(rows), scale, p, seed)
        h = half_step(out_type)
        close(f64(out), want, 1.01 * (2 * U + h) * np.abs(want) + SMALLEST[out_type] / 2, "embed")
        assert (f64(out)[want == 0] == 0).all()
        if layout != "dense":                                  # what lies between the rows stays
            whole = out._base
            assert not whole[:, 1 + dim if layout == "wide" else dim:].any()


def test_embed_zeroes_what_is_dropped_or_padded_whatever_is_there():
    rows = torch.full((4, 64), float("nan"), device="cuda")
    rows[1] = float("inf")
    rows[2] = 1.0
    slots_np = np.array([0, 1, 2, -1, -(1 << 63)], dtype=np.int64)
    out = torch.full((5, 64), 7.0, device="cuda")
    mp.mpzch_embed(torch.from_numpy(slots_np).cuda(), rows, out, scale=2.0, drop_p=0.5, seed=seed_tensor(3))
    kept = ref.keep(5, 64, 0.5, 3)
    got = f64(out)
    assert (got[:3][~kept[:3]] == 0).all() and (got[3:] == 0).all()
    assert np.isnan(got[0][kept[0]]).all() and np.isposinf(got[1][kept[1]]).all() and (got[2][kept[2]] == 4.0).all()
    mp.mpzch_embed(torch.from_numpy(slots_np).cuda(), rows, out, drop_p=1.0, seed=seed_tensor(3))
    assert not out.any()


def test_embed_mask_depends_on_seed_and_position_alone():
    """The mask of (i, j) is the same for every type and alignment, and the share that is dropped is the one asked for:
    of N draws of probability q the share is within 6 sqrt(q (1 - q) / N) of q, but for one seed in 10^8."""
    n, dim, q = 5000, 200, 0.1
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    masks = []
    for dtype, layout in ((F32, "dense"), (BF16, "dense"), (F16, "wide")):
        rng = np.random.Generator(np.random.Philox(key=1))
        rows = tensor2d(rng, 1, dim, dtype, layout)
        rows.fill_(1.0)
        out = tensor2d(rng, n, dim, dtype, layout)
        mp.mpzch_embed(slots, rows, out, drop_p=q, seed=seed_tensor(99))
        masks.append(f64(out) != 0)
    assert (masks[0] == masks[1]).all() and (masks[0] == masks[2]).all()
    assert (masks[0] == ref.keep(n, dim, q, 99)).all()
    assert abs(1 - masks[0].mean() - q) < 6 * math.sqrt(q * (1 - q) / (n * dim))


def test_embed_of_a_table_beyond_32_bits_of_bytes():
    """Rows behind the first 4 GiB, and elements of the output there."""
    num_rows, dim = 20_000_003, 128
    rows = torch.empty(num_rows, dim, dtype=BF16, device="cuda")
    rows[:1000].normal_()
    rows[-1000:].normal_()
    rng = np.random.Generator(np.random.Philox(key=5))
    slots_np = np.concatenate([rng.integers(0, 1000, 3000), num_rows - 1 - rng.integers(0, 1000, 3000)])
    out = torch.empty(6000, dim, dtype=BF16, device="cuda")
    mp.mpzch_embed(torch.from_numpy(slots_np).cuda(), rows, out)
    assert torch.equal(out, rows[torch.from_numpy(slots_np).cuda()])
    del rows, out
    n = 17_000_001
    rows = torch.randn(10, dim, device="cuda").to(BF16)
    slots = torch.arange(n, device="cuda") % 10
    out = torch.empty(n, dim, dtype=BF16, device="cuda")
    mp.mpzch_embed(slots, rows, out)
    assert torch.equal(out[-1000:], rows[slots[-1000:]]) and torch.equal(out[:1000], rows[slots[:1000]])
    assert torch.equal(out.view(-1, 10 * dim // 10)[::1003], rows[slots[::1003]])


# ------------------------------------------------------------------------------------------------ gradient
def run_grad(handle, slots_np, grad, num_rows, out_type, scale, p, seed, cap=None):
    n, dim = grad.shape
    cap = n if cap is None else cap
    out_slots = torch.full((cap + 1,), -77, dtype=torch.int64, device="cuda")
    out_rows = torch.full((cap + 1, dim), -77.0, dtype=out_type, device="cuda")
    count = torch.full((1,), -77, dtype=torch.int64, device="cuda")
    mp.mpzch_embed_grad(handle, torch.from_numpy(slots_np).cuda(), grad, num_rows, out_slots[:cap], out_rows[:cap], count,
                        scale=scale, drop_p=p, seed=seed_tensor(seed))
    return out_slots.cpu().numpy(), out_rows, int(count.item())


def check_grad(handle, slots_np, grad, num_rows, out_type, scale, p, seed, cap=None):
    got_slots, got_rows, count = run_grad(handle, slots_np, grad, num_rows, out_type, scale, p, seed, cap)
    named, total, size, terms = ref.sums(slots_np, f64(grad), num_rows, scale, p, seed)
    cap = len(slots_np) if cap is None else cap
    k = min(cap, len(named))
    assert count == len(named)
    assert np.array_equal(got_slots[:k], named[:k]) and (got_slots[k:] == -77).all()
    rows = f64(got_rows)
    error = 1.01 * (terms[:k, None] + 2) * U * size[:k] + half_step(out_type) * np.abs(total[:k]) * 1.01 + SMALLEST[out_type] / 2
    close(rows[:k], total[:k], error, "grad")
    assert (rows[k:] == f64(torch.full((1,), -77.0, dtype=out_type))[0]).all()      # left as they were


GRAD = [(1, 1, 1, F32, F32), (1, 1000, 16, BF16, BF16), (2, 5, 3, F32, F32), (64, 3, 8, F16, F32), (65, 1 << 20, 64, BF16, F32),
        (255, 255, 100, F32, BF16), (1024, 4096, 16, F32, F32), (2049, 65_535, 50, F16, F16), (4096, 256, 128, BF16, BF16),
        (4097, 255, 333, F32, F32), (1000, 77, 2048, BF16, F32), (300, 50, 4096, F32, F32), (129, 9, 5001, BF16, F32),
        (20_011, 50_021, 48, F32, F32), (65_537, 1_000_000, 64, BF16, F32), (140_001, 65_536, 4, F32, F32),
        (300_007, 6_000_011, 8, BF16, BF16), (9000, (1 << 32) - 2, 32, F32, F32), (3, 2, 1 << 20, BF16, F32)]


@pytest.mark.parametrize("n,num_rows,dim,grad_type,out_type", GRAD)
@pytest.mark.parametrize("kind", ["zipf", "same", "distinct"])
def test_embed_grad(handle, n, num_rows, dim, grad_type, out_type, kind):
    if kind == "distinct" and num_rows > 1 << 21:
        kind = "beyond"
    rng = np.random.Generator(np.random.Philox(key=n * 7 + dim))
    layout = {"zipf": "dense", "same": "wide"}.get(kind, "padded")
    p = 0.25 if dim % 3 else 0.0
    slots_np = draw_slots(rng, n, num_rows, kind)
    grad = tensor2d(rng, n, dim, grad_type, layout, scale=0.1)
    say("grad", n, num_rows, dim, grad_type, out_type, kind, layout, p)
    check_grad(handle, slots_np, grad, num_rows, out_type, 1.5, p, 1234567 + n)


def test_embed_grad_of_nothing_and_of_padding_alone(handle):
    grad = torch.zeros(0, 16, device="cuda")
    _, _, count = run_grad(handle, np.empty(0, np.int64), grad, 10, F32, 1.0, 0.0, 1, cap=4)
    assert count == 0
    for n in (1, 5000):
        grad = torch.full((n, 16), float("nan"), device="cuda")
        check_grad(handle, np.full(n, -1, dtype=np.int64), grad, 10, F32, 1.0, 0.0, 1)


def test_embed_grad_reads_no_padded_and_no_dropped_element(handle):
    rng = np.random.Generator(np.random.Philox(key=8))
    n, dim, p, seed = 3000, 24, 0.5, 4242
    slots_np = draw_slots(rng, n, 200, "zipf")
    grad_np = rng.standard_normal((n, dim)).astype(np.float32)
    clean = torch.from_numpy(grad_np.copy()).cuda()
    grad_np[slots_np < 0] = np.nan
    grad_np[~ref.keep(n, dim, p, seed)] = np.inf
    a = run_grad(handle, slots_np, clean, 200, F32, 1.0, p, seed)
    b = run_grad(handle, slots_np, torch.from_numpy(grad_np).cuda(), 200, F32, 1.0, p, seed)
    assert np.array_equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[2] == b[2]
    check_grad(handle, slots_np, clean, 200, F32, 1.0, 1.0, seed)                   # everything dropped: rows named, sums zero


@pytest.mark.parametrize("cap", [0, 1, 100])
def test_embed_grad_truncates_its_lists(handle, cap):
    rng = np.random.Generator(np.random.Philox(key=9))
    slots_np = draw_slots(rng, 5000, 3000, "zipf")
    check_grad(handle, slots_np, tensor2d(rng, 5000, 20, F32), 3000, F32, 1.0, 0.0, 1, cap=cap)


def test_embed_grad_gives_the_same_bits_again(handle):
    rng = np.random.Generator(np.random.Philox(key=10))
    slots_np = draw_slots(rng, 200_001, 5000, "zipf")
    grad = tensor2d(rng, 200_001, 40, F32)
    a, b = (run_grad(handle, slots_np, grad, 5000, F32, 1.0, 0.1, 5) for _ in range(2))
    assert np.array_equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_embed_grad_of_a_long_batch(handle):
    """More tiles than are added up in place (4 M positions and up); a run that goes through thousands of tiles."""
    n, num_rows, dim = 4_500_001, 1_000_003, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    slots = torch.randint(0, num_rows, (n,), generator=g, device="cuda")
    slots[torch.rand(n, generator=g, device="cuda") < 0.4] = 12345
    grad = torch.randint(-8, 9, (n, dim), generator=g, device="cuda").float()       # sums of whole numbers are exact
    h = mp.mpzch_embed_create()
    out_slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    out_rows = torch.zeros(n, dim, device="cuda")
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    mp.mpzch_embed_grad(h, slots, grad, num_rows, out_slots, out_rows, count)
    named, total, _, _ = ref.sums(slots.cpu().numpy(), f64(grad), num_rows, 1.0, 0.0, 0)
    k = int(count.item())
    assert k == len(named) and np.array_equal(out_slots[:k].cpu().numpy(), named)
    assert np.array_equal(f64(out_rows[:k]), total)
    mp.mpzch_embed_destroy(h)


RUNS = [1, 1, 2, 3, 5, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 160, 191, 192, 193, 255, 256, 257, 258, 300, 383, 384, 385, 511, 512, 513,
        640, 1000, 1024, 1025, 2047, 2048, 2049, 2175, 2176, 2177, 2178, 4000]


@pytest.mark.parametrize("dim,dtype", [(1, F32), (2, BF16), (16, F32), (64, BF16), (130, F32), (512, BF16), (513, F32), (1024, BF16), (2056, BF16)])
@pytest.mark.parametrize("order", ["up", "down", "mixed", "short"])
def test_sums_of_runs_of_every_length(handle, dim, dtype, order):
    """Runs that end and begin at, before and behind the borders of parts, tiles and what lies behind them; sums of small whole
    numbers are exact, so the results of gradient and step are, too."""
    rng = np.random.Generator(np.random.Philox(key=dim * 10 + len(order)))
    lengths = {"up": RUNS, "down": RUNS[::-1], "mixed": list(rng.permutation(RUNS + [1] * 300 + [2] * 100)), "short": RUNS[:16] * 3}[order]
    if dim > 600:
        lengths = [x for x in lengths if x < 1100]
    slots_np = np.repeat(np.arange(len(lengths)) * 3 + 1, lengths).astype(np.int64)
    n, num_rows = len(slots_np), 3 * len(lengths) + 2
    slots_np = slots_np[rng.permutation(n)]
    grad_np = rng.integers(-4, 5, size=(n, dim)).astype(np.float32)
    grad = torch.from_numpy(grad_np).cuda().to(dtype)
    say("runs", n, num_rows, dim, dtype, order)
    got_slots, got_rows, count = run_grad(handle, slots_np, grad, num_rows, F32, 1.0, 0.0, 0)
    named, total, _, _ = ref.sums(slots_np, grad_np, num_rows, 1.0, 0.0, 0)
    assert count == len(named) and np.array_equal(got_slots[:count], named)
    assert np.array_equal(f64(got_rows)[:count], total) and (f64(got_rows)[count:] == -77).all()
    if dim > 1024:
        return
    rows = torch.zeros(num_rows, dim, device="cuda")             # SGD with a rate of 1 / 2 from zero: -total / 2
    mp.mpzch_embed_step(handle, torch.from_numpy(slots_np).cuda(), grad, rows, None, torch.full((1,), 0.5, device="cuda"))
    want = np.zeros((num_rows, dim))
    want[named] = -0.5 * total
    assert np.array_equal(f64(rows), want)


@pytest.mark.parametrize("n,num_rows", [(8192, 100), (8193, 100), (65_536, 70_000), (65_537, 70_000), (70_001, (1 << 32) - 2),
                                        (524_288, 1 << 20), (524_289, 1 << 20), (1_048_576, 33), (1_048_577, 33_000_000), (2_100_000, 7)])
def test_gradients_of_every_way_to_sort(handle, n, num_rows):
    """Sizes on both sides of where another sort takes over; whole numbers again."""
    rng = np.random.Generator(np.random.Philox(key=n))
    slots_np = draw_slots(rng, n, num_rows, "zipf")
    grad_np = rng.integers(-8, 9, size=(n, 2)).astype(np.float32)
    say("sort", n, num_rows)
    got_slots, got_rows, count = run_grad(handle, slots_np, torch.from_numpy(grad_np).cuda(), num_rows, F32, 1.0, 0.0, 0)
    named, total, _, _ = ref.sums(slots_np, grad_np, num_rows, 1.0, 0.0, 0)
    assert count == len(named) and np.array_equal(got_slots[:count], named)
    assert np.array_equal(f64(got_rows)[:count], total)


def test_scratch_grows_and_keeps_what_it_had_room_for():
    """A handle that is used before anything is reserved, then for longer batches and rows, then for short ones again."""
    h = mp.mpzch_embed_create()
    rng = np.random.Generator(np.random.Philox(key=21))
    for n, dim in ((10, 4), (5000, 4), (100, 700), (70_000, 12), (3, 3000), (70_000, 16), (1, 1)):
        check_grad(h, draw_slots(rng, n, 50, "zipf"), tensor2d(rng, n, dim, F32), 50, F32, 1.0, 0.0, 0)
    mp.mpzch_embed_destroy(h)


def test_sums_of_gradients_and_tables_beyond_32_bits_of_bytes():
    """Gradient rows and table rows behind the first 4 GiB; whole numbers, whose sums are exact."""
    n, dim, num_rows = 8_700_001, 256, 1009
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    grad = torch.randint(-3, 4, (n, dim), generator=g, device="cuda", dtype=torch.int8).to(BF16)
    slots = torch.randint(0, num_rows, (n,), generator=g, device="cuda")
    want = torch.zeros(num_rows, dim, device="cuda")
    for at in range(0, n, 1 << 20):
        want.index_add_(0, slots[at:at + (1 << 20)], grad[at:at + (1 << 20)].float())
    h = mp.mpzch_embed_create()
    out_slots = torch.zeros(num_rows, dtype=torch.int64, device="cuda")
    out_rows, count = torch.zeros(num_rows, dim, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    mp.mpzch_embed_grad(h, slots, grad, num_rows, out_slots, out_rows, count)
    assert int(count.item()) == num_rows and torch.equal(out_slots, torch.arange(num_rows, device="cuda"))
    assert torch.equal(out_rows, want)
    del grad
    many = 10_000_019
    rows, far = torch.zeros(many, 128, device="cuda"), many - 1 - torch.arange(3000, device="cuda") * 3
    slots, grad = far.repeat(4), torch.randint(-3, 4, (12_000, 128), generator=g, device="cuda").float()
    mp.mpzch_embed_step(h, slots, grad, rows, None, torch.ones(1, device="cuda"))
    assert torch.equal(rows[far], -grad.view(4, 3000, 128).sum(0))
    rows[far] = 0
    assert not rows.any()
    mp.mpzch_embed_destroy(h)


def test_embed_grad_against_differences(handle):
    """The derivative of <c, embed(rows)> in the direction d is <G, d>: the lookup is linear, so the difference quotient over a
    step of 1 has only the roundings of the two lookups: 2 (2 u) sum |c| f (|w| + |d|), and the gradient's."""
    rng = np.random.Generator(np.random.Philox(key=11))
    n, num_rows, dim, p, seed, scale = 700, 90, 36, 0.3, 77, 1.25
    slots_np = draw_slots(rng, n, num_rows, "zipf")
    slots = torch.from_numpy(slots_np).cuda()
    w, d = tensor2d(rng, num_rows, dim, F32), tensor2d(rng, num_rows, dim, F32)
    c = tensor2d(rng, n, dim, F32)
    a, b = torch.empty(n, dim, device="cuda"), torch.empty(n, dim, device="cuda")
    mp.mpzch_embed(slots, w, a, scale=scale, drop_p=p, seed=seed_tensor(seed))
    moved = w + d
    mp.mpzch_embed(slots, moved, b, scale=scale, drop_p=p, seed=seed_tensor(seed))
    quotient = float((f64(c) * (f64(b) - f64(a))).sum())
    got_slots, got_rows, k = run_grad(handle, slots_np, c, num_rows, F32, scale, p, seed)
    real_d = f64(moved) - f64(w)                                 # the direction that the rounded sum really went
    along = float((f64(got_rows)[:k] * real_d[got_slots[:k]]).sum())
    there = slots_np >= 0
    f = ref.factor(scale, p)
    size = (np.abs(f64(c)[there]) * f * (np.abs(f64(w)) + np.abs(f64(moved)))[slots_np[there]]).sum()
    _, _, sizes, terms = ref.sums(slots_np, f64(c), num_rows, scale, p, seed)
    error = 2 * U * size + ((terms[:, None] + 3) * U * sizes * np.abs(real_d[got_slots[:k]])).sum()
    assert abs(quotient - along) <= 1.01 * error, (quotient, along, error)


# ------------------------------------------------------------------------------------------------ step
STEP = [(1, 1, 1, F32, F32), (1, 1000, 16, BF16, BF16), (64, 3, 8, F16, F32), (1024, 4096, 16, F32, F32), (2049, 65_535, 50, F16, F16),
        (4097, 255, 333, F32, F32), (1000, 77, 1024, BF16, BF16), (500, 60, 1001, F32, BF16), (3000, 4099, 1023, BF16, F32),
        (20_011, 50_021, 48, F32, F32), (65_537, 1_000_000, 64, BF16, F32), (140_001, 4096, 4, F32, F32), (777, 30, 600, BF16, F32)]


@pytest.mark.parametrize("n,num_rows,dim,grad_type,table", STEP)
@pytest.mark.parametrize("kind", ["zipf", "same", "distinct"])
@pytest.mark.parametrize("rule", ["sgd", "adagrad"])
def test_embed_step(handle, n, num_rows, dim, grad_type, table, kind, rule):
    rng = np.random.Generator(np.random.Philox(key=n * 11 + dim))
    layout = {"zipf": "dense", "same": "wide"}.get(kind, "padded")
    p, scale, lr, eps, seed = (0.25 if dim % 3 else 0.0), 0.75, float(np.float32(0.05)), float(np.float32(1e-6)), 31 + n
    slots_np = draw_slots(rng, n, num_rows, kind)
    grad = tensor2d(rng, n, dim, grad_type, layout, scale=0.1)
    rows = tensor2d(rng, num_rows, dim, table, layout)
    state = torch.from_numpy(rng.random(num_rows).astype(np.float32)).cuda() if rule == "adagrad" else None
    if state is not None:
        state[::2] = 0                                           # rows that have seen nothing yet
    before, state_before = rows.clone(), None if state is None else state.clone()
    say("step", n, num_rows, dim, grad_type, table, kind, rule, layout, p)
    mp.mpzch_embed_step(handle, torch.from_numpy(slots_np).cuda(), grad, rows, state, torch.full((1,), lr, device="cuda"), eps,
                        scale=scale, drop_p=p, seed=seed_tensor(seed))
    named, total, size, terms = ref.sums(slots_np, f64(grad), num_rows, scale, p, seed)
    w0 = f64(before)
    want, want_state = ref.step(w0, None if state is None else f64(state_before), named, total, lr, eps)
    untouched = np.setdiff1d(np.arange(num_rows), named)
    assert torch.equal(rows[torch.from_numpy(untouched).cuda()], before[torch.from_numpy(untouched).cuda()])
    e_g = (terms[:, None] + 2) * U * size
    h = half_step(table)
    change = np.abs(want[named] - w0[named])
    if rule == "sgd":
        error = lr * e_g + 4 * U * (np.abs(w0[named]) + change) + h * np.abs(want[named])
    else:
        assert torch.equal(state[torch.from_numpy(untouched).cuda()], state_before[torch.from_numpy(untouched).cuda()])
        e_state, e_change = adagrad_errors(total, e_g, f64(state_before)[named], want_state[named], lr, eps)
        close(f64(state)[named], want_state[named], 1.01 * e_state + SMALLEST[F32], "state")
        error = e_change + 4 * U * (np.abs(w0[named]) + change) + h * np.abs(want[named])
    close(f64(rows)[named], want[named], 1.01 * error + SMALLEST[table], "step")
    if layout != "dense":
        assert not rows._base[:, 1 + dim if layout == "wide" else dim:].any()


def test_embed_step_of_dropped_gradients_changes_nothing(handle):
    """Sums of zero: 0 / (sqrt(0) + eps) = 0."""
    rows = torch.randn(50, 32, device="cuda")
    before, state = rows.clone(), torch.zeros(50, device="cuda")
    slots = torch.arange(50, device="cuda")
    grad = torch.full((50, 32), float("inf"), device="cuda")
    mp.mpzch_embed_step(handle, slots, grad, rows, state, torch.ones(1, device="cuda"), 1e-8, drop_p=1.0, seed=seed_tensor(1))
    mp.mpzch_embed_step(handle, slots[:0], grad[:0], rows, state, torch.ones(1, device="cuda"), 1e-8)
    mp.mpzch_embed_step(handle, slots - 60, grad, rows, None, torch.ones(1, device="cuda"))
    assert torch.equal(rows, before) and not state.any()


# ------------------------------------------------------------------------------------------------ together
def test_a_training_loop_on_a_table(handle):
    """Remap, lookup with dropout, gradient of sum(out^2) / 2 for out, step, reset of evicted rows and of their state, as a program
    has them one behind the other on a stream of its own; every step against the formulas."""
    dim, lr, eps, p = 32, 0.1, 1e-6, 0.2
    t = mp.MpzchTable(3000, 16, mp.EVICT_TTL, 2, 99)
    rng = np.random.Generator(np.random.Philox(key=12))
    rows = torch.from_numpy(rng.standard_normal((3000, dim)).astype(np.float32)).cuda()
    state = torch.zeros(3000, device="cuda")
    lr_dev = torch.full((1,), lr, device="cuda")
    init = torch.full((dim,), 0.5, device="cuda")
    seed = seed_tensor(1000)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    evictions = 0
    with torch.cuda.stream(stream):
        for k in range(6):
            ids_np = np.concatenate([wl.zipf_ids(rng, 1500, 1.1, 4000), wl.rank_to_id(rng.integers(10_000 * (k + 1), 10_000 * (k + 2), 700))])
            slots = t.remap(torch.from_numpy(ids_np).cuda(), k)
            mp.mpzch_reset_rows(t._evicted, t.num_evicted, rows, init)
            mp.mpzch_reset_rows(t._evicted, t.num_evicted, state.view(-1, 1))
            w0, s0 = f64(rows), f64(state)
            out = torch.empty(len(ids_np), dim, device="cuda")
            mp.mpzch_embed(slots, rows, out, scale=1.0, drop_p=p, seed=seed)
            mp.mpzch_embed_step(handle, slots, out, rows, state, lr_dev, eps, drop_p=p, seed=seed)
            slots_np, evicted = slots.cpu().numpy(), t.evicted.cpu().numpy()
            evictions += len(evicted)
            if len(evicted):
                fresh = np.setdiff1d(evicted, [])
                assert (w0[fresh] == 0.5).all() and (s0[fresh] == 0).all()
            want_out = ref.embed(slots_np, w0, 1.0, p, 1000 + k)
            close(f64(out), want_out, 1.01 * 3 * U * np.abs(want_out), "out")
            named, total, size, terms = ref.sums(slots_np, f64(out), 3000, 1.0, p, 1000 + k)
            want, want_state = ref.step(w0, s0, named, total, float(np.float32(lr)), eps)
            # (tolerances of test_embed_step)
            e_g = (terms[:, None] + 2) * U * size
            e_state, e_change = adagrad_errors(total, e_g, s0[named], want_state[named], float(np.float32(lr)), eps)
            close(f64(state)[named], want_state[named], 1.01 * e_state + SMALLEST[F32], "state")
            error = e_change + 5 * U * (np.abs(w0[named]) + np.abs(want - w0)[named])
            close(f64(rows)[named], want[named], 1.01 * error, "rows")
            seed += 1
    assert evictions > 0
    t.close()


def test_captured_lookup_gradient_and_step_replay(handle):
    """One graph of the three operators, replayed with new slots, gradients, rates and seeds in the same buffers, eager work and
    synchronisation between the replays; every replay has the bits of the eager calls."""
    n, num_rows, dim, p = 5000, 2000, 24, 0.1
    h = mp.mpzch_embed_create()
    mp.mpzch_embed_reserve(h, n, dim)
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    grad = torch.zeros(n, dim, device="cuda").to(BF16)
    seed, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")

    def buffers():
        return dict(rows=torch.zeros(num_rows, dim, device="cuda"), state=torch.zeros(num_rows, device="cuda"),
                    out=torch.zeros(n, dim, device="cuda").to(BF16), out_slots=torch.zeros(n, dtype=torch.int64, device="cuda"),
                    out_rows=torch.zeros(n, dim, device="cuda"), count=torch.zeros(1, dtype=torch.int64, device="cuda"))

    def calls(which, b):
        mp.mpzch_embed(slots, b["rows"], b["out"], scale=2.0, drop_p=p, seed=seed)
        mp.mpzch_embed_grad(which, slots, grad, num_rows, b["out_slots"], b["out_rows"], b["count"], drop_p=p, seed=seed)
        mp.mpzch_embed_step(which, slots, grad, b["rows"], b["state"], lr, 1e-6, drop_p=p, seed=seed)

    captured, eager = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(h, captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(h, captured)
    rng = np.random.Generator(np.random.Philox(key=13))
    for k in range(4):
        kind = ["zipf", "same", "distinct", "padding"][k]
        s = draw_slots(rng, n, num_rows, kind)
        slots.copy_(torch.from_numpy(s).cuda())
        grad.copy_(tensor2d(rng, n, dim, BF16))
        seed.fill_(100 + k)
        lr.fill_(0.1 / (k + 1))
        fresh = tensor2d(rng, num_rows, dim, F32)
        for b in (captured, eager):
            b["rows"].copy_(fresh)
            b["state"].fill_(0.25)
            for name in ("out", "out_slots", "out_rows", "count"):
                b[name].zero_()
        say("replay", k, kind)
        graph.replay()
        torch.cuda.synchronize()
        calls(handle, eager)
        torch.cuda.synchronize()
        for name in captured:
            assert torch.equal(captured[name], eager[name]), (name, kind)
    del graph
    mp.mpzch_embed_destroy(h)


def test_two_handles_on_two_streams_do_not_meet():
    rng = np.random.Generator(np.random.Philox(key=14))
    work = []
    for k in range(2):
        s = draw_slots(rng, 50_000, 3000, "zipf")
        work.append(dict(h=mp.mpzch_embed_create(), s=s, slots=torch.from_numpy(s).cuda(), grad=tensor2d(rng, 50_000, 16, F32),
                         stream=torch.cuda.Stream(), out_slots=torch.zeros(50_000, dtype=torch.int64, device="cuda"),
                         out_rows=torch.zeros(50_000, 16, device="cuda"), count=torch.zeros(1, dtype=torch.int64, device="cuda")))
        mp.mpzch_embed_reserve(work[k]["h"], 50_000, 16)
    torch.cuda.synchronize()
    for _ in range(3):
        for w in work:
            with torch.cuda.stream(w["stream"]):
                mp.mpzch_embed_grad(w["h"], w["slots"], w["grad"], 3000, w["out_slots"], w["out_rows"], w["count"])
    torch.cuda.synchronize()
    for w in work:
        named, total, size, terms = ref.sums(w["s"], f64(w["grad"]), 3000, 1.0, 0.0, 0)
        k = int(w["count"].item())
        assert k == len(named) and np.array_equal(w["out_slots"][:k].cpu().numpy(), named)
        close(f64(w["out_rows"][:k]), total, 1.01 * (terms[:, None] + 3) * U * size, "grad")
        mp.mpzch_embed_destroy(w["h"])


def test_binding_refuses_tensors_that_do_not_fit(handle):
    slots = torch.zeros(8, dtype=torch.int64, device="cuda")
    rows, out = torch.zeros(10, 16, device="cuda"), torch.zeros(8, 16, device="cuda")
    count, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda")
    refused = pytest.raises(AssertionError)
    for bad in ((slots.int(), rows, out), (slots, rows.double(), out), (slots, rows, out[:7]), (slots, rows, out[:, :8]),
                (slots, rows.cpu(), out), (slots, rows.t(), out), (slots[::2], rows, out[:4]), (slots, rows[0], out),
                (slots, rows[:1].expand(10, 16), out)):
        with refused:
            mp.mpzch_embed(*bad)
    with refused:
        mp.mpzch_embed(slots, rows, out, drop_p=0.1, seed=torch.zeros(2, dtype=torch.int64, device="cuda"))
    for bad in ((slots, out[:7], 10, slots, out, count), (slots, out, 10, slots[:7], out, count),
                (slots, out, 10, slots, out, None), (slots, out, 10, slots, out[:, :8], count)):
        with refused:
            mp.mpzch_embed_grad(handle, *bad)
    for bad in ((slots, out, rows, torch.zeros(9, device="cuda"), lr), (slots, out[:, :8], rows, None, lr),
                (slots, out, rows, None, torch.ones(1, device="cuda").double())):
        with refused:
            mp.mpzch_embed_step(handle, *bad)
    for p, scale in ((0.5, 1.0), (-0.1, 1.0), (1.1, 1.0), (float("nan"), 1.0), (0.0, float("inf"))):
        with pytest.raises(mp.MpzchError) as e:                  # (the first: dropout without a seed)
            mp.mpzch_embed(slots, rows, out, scale=scale, drop_p=p)
        assert e.value.status == 1
    assert not out.any() and not rows.any()


# ------------------------------------------------------------------------------------------------ what went wrong before
@pytest.mark.parametrize("dim,dtype", [(1025, BF16), (2048, BF16), (4100, F32), (16_384, BF16)])
def test_long_runs_of_rows_of_many_column_blocks_go_to_their_own_place(dim, dtype):
    """Rows of more than 1 024 elements are shared out over workgroups by columns, and each of them joins its columns of a long run by
    itself.  Where the run is in the list changes from call to call on one handle, from a scratch that nothing has used on: every
    block of columns has to take this call's place.  Sums of small whole numbers are exact."""
    rng = np.random.Generator(np.random.Philox(key=dim))
    n, num_rows = 4500, 9000
    h = mp.mpzch_embed_create()
    for k, single in enumerate((0, 700, 3, 250, 1500, 0)):      # rows of one position in front of the long runs
        long_rows = 2000 + 7 * np.arange(3) + k
        lengths = np.array([1100, 900, n - single - 2000])
        slots_np = np.concatenate([np.arange(single), np.repeat(long_rows, lengths)]).astype(np.int64)
        slots_np = slots_np[rng.permutation(n)]
        grad_np = rng.integers(-4, 5, size=(n, dim)).astype(np.float32)
        say("long runs", dim, dtype, k, single)
        got_slots, got_rows, count = run_grad(h, slots_np, torch.from_numpy(grad_np).cuda().to(dtype), num_rows, F32, 1.0, 0.0, 0, cap=2000)
        named, total, _, _ = ref.sums(slots_np, grad_np, num_rows, 1.0, 0.0, 0)
        assert count == len(named) == single + 3 and np.array_equal(got_slots[:count], named)
        assert np.array_equal(f64(got_rows)[:count], total) and (f64(got_rows)[count:] == -77).all()
    mp.mpzch_embed_destroy(h)


@pytest.mark.parametrize("dim", [1, 16, 50, 600])
@pytest.mark.parametrize("lr,eps,state_exp,grad_exp", [
    (1.0, 2.0 ** -149, None, None), (0.5, 1e-44, None, None), (1e30, 1e-10, None, None), (0.0, 2.0 ** -149, None, None),
    (1e30, 1e-12, -60, -40), (2.0 ** 127, 2.0 ** -126, -60, -60), (1e-30, 1e-6, 60, 40), (-1e30, 1e-12, -60, -40)])
def test_rates_beyond_32_bit_floats(handle, dim, lr, eps, state_exp, grad_exp):
    """lr / (sqrt(state) + eps) need not fit 32 bits where lr G / (sqrt(state) + eps) does.  Sums of zero (terms of zero, terms that
    cancel, everything dropped) change nothing, whatever lr and eps; others change the rows by what the formula says.  Rows of one
    position, of a few, and of thousands, which a whole workgroup adds up.

    With a sum G of terms of absolute sum S: tolerances of the step above, from weights of zero; the change stays above 2^-126."""
    rng = np.random.Generator(np.random.Philox(key=dim))
    lr, eps = float(np.float32(lr)), float(np.float32(eps))
    slots_np = np.concatenate([np.arange(40), np.repeat([50, 51], 30), np.repeat([60, 61], 2600)]).astype(np.int64)
    n, num_rows = len(slots_np), 64
    zero = state_exp is None
    grad_np = rng.integers(1, 5, size=(n, dim)).astype(np.float64) * 2.0 ** (0 if zero else grad_exp)
    if zero:
        grad_np[:40] = 0
        grad_np[1::2] = -grad_np[::2]                            # (pairs of neighbours, which are of one row)
    order = rng.permutation(n)
    slots_np, grad_np = slots_np[order], grad_np[order]
    grad = torch.from_numpy(grad_np).cuda().float()
    rows = torch.from_numpy(rng.standard_normal((num_rows, dim)) if zero else np.zeros((num_rows, dim))).cuda().float()
    state = torch.full((num_rows,), 0.0 if zero else 2.0 ** state_exp, device="cuda")
    before, state_before = rows.clone(), state.clone()
    say("rates", dim, lr, eps, state_exp)
    mp.mpzch_embed_step(handle, torch.from_numpy(slots_np).cuda(), grad, rows, state, torch.full((1,), lr, device="cuda"), eps)
    if zero:
        assert torch.equal(rows, before) and torch.equal(state, state_before)
        mp.mpzch_embed_step(handle, torch.from_numpy(slots_np).cuda(), torch.full_like(grad, 3.0), rows, state,
                            torch.full((1,), lr, device="cuda"), eps, drop_p=1.0, seed=seed_tensor(5))
        assert torch.equal(rows, before) and torch.equal(state, state_before)
        return
    named, total, size, terms = ref.sums(slots_np, f64(grad), num_rows, 1.0, 0.0, 0)
    want, want_state = ref.step(f64(before), f64(state_before), named, total, lr, eps)
    e_g = (terms[:, None] + 2) * U * size
    e_state, e_change = adagrad_errors(total, e_g, f64(state_before)[named], want_state[named], abs(lr), eps)
    assert (np.abs(want[named]) > 2.0 ** -126).all() and (np.abs(want[named]) < 2.0 ** 127).all()
    close(f64(state)[named], want_state[named], 1.01 * e_state, "state")
    close(f64(rows)[named], want[named], 1.01 * (e_change + 5 * U * np.abs(want[named])), "rows")


def test_lookup_and_gradient_refuse_to_lose_a_gradient(handle):
    """Neither is differentiable by itself: with gradients enabled, rows or gradients that require one are refused, not detached
    in silence.  Without (torch.no_grad(), detach(), the inside of an autograd function) the same tensors do."""
    slots = torch.tensor([1, 0, 1], device="cuda")
    weight = torch.nn.Parameter(torch.randn(4, 8, device="cuda"))
    out, count = torch.zeros(3, 8, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    with pytest.raises(AssertionError, match="gradient"):
        mp.mpzch_embed(slots, weight, out)
    with pytest.raises(AssertionError, match="gradient"):
        mp.mpzch_embed(slots, weight * 2, out)
    out_slots, out_rows = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, 8, device="cuda")
    needs = torch.ones(3, 8, device="cuda", requires_grad=True)
    with pytest.raises(AssertionError, match="gradient"):
        mp.mpzch_embed_grad(handle, slots, needs, 4, out_slots, out_rows, count)
    assert not out.any() and not count.any()
    mp.mpzch_embed(slots, weight.detach(), out)
    assert torch.equal(out, weight[slots])
    out.zero_()
    with torch.no_grad():
        mp.mpzch_embed(slots, weight, out)
        mp.mpzch_embed_grad(handle, slots, needs, 4, out_slots, out_rows, count)
    assert torch.equal(out, weight[slots]) and int(count.item()) == 2

    class Lookup(torch.autograd.Function):
        @staticmethod
        def forward(ctx, rows, at):
            ctx.save_for_backward(at)
            ctx.shape = rows.shape
            result = torch.empty(at.numel(), rows.shape[1], device="cuda")
            mp.mpzch_embed(at, rows, result, scale=2.0)
            return result

        @staticmethod
        def backward(ctx, g):
            (at,) = ctx.saved_tensors
            named = torch.zeros(at.numel(), dtype=torch.int64, device="cuda")
            sums, k = torch.zeros(at.numel(), ctx.shape[1], device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
            mp.mpzch_embed_grad(handle, at, g.contiguous(), ctx.shape[0], named, sums, k, scale=2.0)
            whole = torch.zeros(ctx.shape, device="cuda")
            m = int(k.item())
            whole[named[:m]] = sums[:m]
            return whole, None

    c = torch.randint(-3, 4, (3, 8), device="cuda").float()
    (Lookup.apply(weight, slots) * c).sum().backward()
    want = torch.zeros(4, 8, device="cuda").index_add_(0, slots, 2 * c)
    assert torch.equal(weight.grad, want)


def test_what_is_written_gets_a_new_version(handle):
    """Autograd notices that a tensor which it keeps for a backward pass was written over."""
    slots = torch.tensor([1, 0, 1], device="cuda")
    rows, state, lr = torch.randn(4, 8, device="cuda"), torch.zeros(4, device="cuda"), torch.ones(1, device="cuda")
    out, count = torch.zeros(3, 8, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    out_slots, out_rows = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, 8, device="cuda")
    read = (slots, lr)
    read_before = [t._version for t in read]
    for call, written in ((lambda: mp.mpzch_embed(slots, rows, out), (out,)),
                          (lambda: mp.mpzch_embed_grad(handle, slots, out, 4, out_slots, out_rows, count), (out_slots, out_rows, count)),
                          (lambda: mp.mpzch_embed_step(handle, slots, out, rows, state, lr), (rows, state)),
                          (lambda: mp.mpzch_embed_step(handle, slots, out, rows, None, lr), (rows,))):
        before = [t._version for t in written]
        call()
        assert all(t._version > b for t, b in zip(written, before))
    assert [t._version for t in read] == read_before
    weight = torch.randn(4, 8, device="cuda", requires_grad=True)
    loss = (weight * weight).sum()                               # (keeps the weight)
    mp.mpzch_embed_step(handle, slots, out, weight, None, lr)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        kept = torch.zeros(3, 8, device="cuda")
    mp.mpzch_embed(slots, rows, kept)                            # (tensors of inference mode have no version)
    assert torch.equal(kept, rows[slots])


def fenced(n, dim, dtype, values=None):
    """(the whole tensor, n x dim of it): rows that begin at the fourth element of wider ones, with a sentinel in front of, between and
    behind them that none of the operators writes"""
    whole = torch.full((n + 2, dim + 7), 1536.0, dtype=dtype, device="cuda")
    view = whole[1:-1, 3:3 + dim]
    if values is not None:
        view.copy_(values)
    return whole, view


def assert_fence_stands(whole, dim):
    inside = torch.zeros_like(whole, dtype=torch.bool)
    inside[1:-1, 3:3 + dim] = True
    assert bool((whole.float()[~inside] == 1536.0).all())


@pytest.mark.parametrize("dim", [1, 2, 3, 5, 7, 8, 9, 15, 50, 129, 511, 1001, 1024, 1025, 2051])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_nothing_in_front_of_or_behind_the_rows_is_touched(handle, dim, dtype):
    """The last piece of a row whose length is no multiple of a piece is moved back towards the row's begin; padding and dropped elements
    write zeros.  Neither reaches beyond the row, and single rows, of some positions and of thousands, are where they should be."""
    rng = np.random.Generator(np.random.Philox(key=dim))
    n, num_rows = 3000, 300
    slots_np = draw_slots(rng, n, num_rows, "zipf")
    slots_np[:1200] = 7
    slots_np[5] = -1
    slots_np = slots_np[rng.permutation(n)]
    slots = torch.from_numpy(slots_np).cuda()
    table = rng.integers(-8, 9, size=(num_rows, dim)).astype(np.float32)
    whole_rows, rows = fenced(num_rows, dim, dtype, torch.from_numpy(table))
    whole_out, out = fenced(n, dim, dtype)
    say("fence", dim, dtype)
    mp.mpzch_embed(slots, rows, out, scale=2.0, drop_p=0.5, seed=seed_tensor(6))
    assert np.array_equal(f64(out), ref.embed(slots_np, table.astype(np.float64), 2.0, 0.5, 6))
    assert_fence_stands(whole_out, dim)
    assert_fence_stands(whole_rows, dim)
    grad_np = rng.integers(-1, 2, size=(n, dim)).astype(np.float32)
    whole_grad, grad = fenced(n, dim, dtype, torch.from_numpy(grad_np))
    sums = torch.full((num_rows + 2, dim), 1536.0, device="cuda")
    named, total, _, _ = ref.sums(slots_np, grad_np, num_rows, 1.0, 0.5, 6)
    out_slots, count = torch.zeros(num_rows, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    mp.mpzch_embed_grad(handle, slots, grad, num_rows, out_slots, sums[1:-1], count, drop_p=0.5, seed=seed_tensor(6))
    k = int(count.item())
    assert k == len(named) and np.array_equal(out_slots[:k].cpu().numpy(), named) and np.array_equal(f64(sums)[1:1 + k], total)
    assert bool((sums[0] == 1536.0).all()) and bool((sums[1 + k:] == 1536.0).all())
    assert_fence_stands(whole_grad, dim)
    if dim > 1024:
        return
    state = torch.full((num_rows + 2,), 1536.0, device="cuda")
    state[1:-1] = 0
    for s in (None, state[1:-1]):
        mp.mpzch_embed_step(handle, slots, grad, rows, s, torch.full((1,), 0.5, device="cuda"), 1e-6, drop_p=0.5, seed=seed_tensor(6))
        assert_fence_stands(whole_rows, dim)
    assert float(state[0]) == 1536.0 and float(state[-1]) == 1536.0
    untouched = np.setdiff1d(np.arange(num_rows), named)
    assert np.array_equal(f64(rows)[untouched], table[untouched]) and not f64(state)[1:-1][untouched].any()
