"""The operators between a table's slots and a model: typed lookup of embedding rows with scaling and dropout, its gradient by
sorted slots, and the optimizer step of the rows that a batch touched, as cases that can be timed and compared.

  embed  out[i, j] = f * rows[slot_i mod num_rows, j] where the mask keeps (i, j), else 0; a negative slot is padding: zeros
  grad   for every row that is named, ascending: f * sum of the kept grad[i, j] of its positions i
  step   the same sums G, applied: SGD  w -= lr G,  or row-wise Adagrad  s += mean_j G^2,  w -= lr G / (sqrt(s) + eps)

The mask is never stored: 64-bit word i * ceil(dim / 4) + j / 4 of the SplitMix64 stream that starts at the seed holds the 16-bit
draws of four neighbouring elements; an element is dropped where its draw is below T = floor(65536 p + 1/2), and what is kept
grows by 65536 / (65536 - T), which is in f beside the scale.

With `own` false, run() computes this from elementary torch operations; with `own` true it calls the framework.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEVICE = "cuda"
DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
GOLDEN = 0x9E3779B97F4A7C15
MIX = (0xBF58476D1CE4E5B9, 0x94D049BB133111EB)
LR, EPS = 0.02, 1e-6


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # serving, one token at a time: a single row on its way into the first layer
        dict(name="embed one", op="embed", n=1, rows=1_000_000, dim=128, table="bfloat16", grad="bfloat16", drop=0.0, pad=0.0,
             alpha=1.05, scatter=True, rule=""),
        # a training batch of the medium table, dropout after the embedding, activations in 16 bits, some positions padded
        dict(name="embed batch", op="embed", n=65536, rows=1_000_000, dim=64, table="float32", grad="bfloat16", drop=0.1, pad=0.02,
             alpha=1.05, scatter=True, rule=""),
        # token ids of a vocabulary (small ids are the frequent ones), long rows, a ragged number of tokens
        dict(name="embed vocabulary", op="embed", n=8191, rows=50_021, dim=2048, table="bfloat16", grad="bfloat16", drop=0.1,
             pad=0.0, alpha=1.1, scatter=False, rule=""),
        # a step of the large shard: 2 M positions, rows of 256 bytes out of 6.4 GB
        dict(name="embed shard", op="embed", n=2_000_000, rows=25_000_000, dim=128, table="bfloat16", grad="bfloat16", drop=0.1,
             pad=0.0, alpha=1.05, scatter=True, rule=""),
        # the tiniest training step: launches are all that counts
        dict(name="grad tiny", op="grad", n=1024, rows=4096, dim=16, table="float32", grad="float32", drop=0.0, pad=0.0,
             alpha=1.1, scatter=True, rule=""),
        # no size a round number, half-precision gradients, a fifth of the batch padding
        dict(name="grad ragged", op="grad", n=20_011, rows=50_021, dim=50, table="float32", grad="float16", drop=0.2, pad=0.2,
             alpha=1.1, scatter=True, rule=""),
        # strongly skewed ids: the most frequent one is a fifth of the batch
        dict(name="grad skewed", op="grad", n=300_007, rows=6_000_011, dim=64, table="float32", grad="bfloat16", drop=0.0, pad=0.0,
             alpha=1.2, scatter=True, rule=""),
        # the gradient of the large shard's lookup, its sums kept in 32 bits for an exchange between GPUs
        dict(name="grad shard", op="grad", n=2_000_000, rows=25_000_000, dim=128, table="float32", grad="bfloat16", drop=0.1,
             pad=0.0, alpha=1.05, scatter=True, rule=""),
        # SGD on a small table
        dict(name="step tiny", op="step", n=1024, rows=4096, dim=16, table="float32", grad="float32", drop=0.0, pad=0.0,
             alpha=1.1, scatter=True, rule="sgd"),
        # a training batch of the medium table, row-wise Adagrad, the mask of "embed batch" again
        dict(name="step batch", op="step", n=65536, rows=1_000_000, dim=64, table="float32", grad="bfloat16", drop=0.1, pad=0.02,
             alpha=1.05, scatter=True, rule="adagrad"),
        # long rows of a vocabulary in 16 bits
        dict(name="step vocabulary", op="step", n=16_384, rows=50_021, dim=1024, table="bfloat16", grad="bfloat16", drop=0.0,
             pad=0.0, alpha=1.1, scatter=False, rule="adagrad"),
        # a million positions on a table of a few million rows
        dict(name="step shard", op="step", n=1_000_000, rows=6_000_011, dim=128, table="bfloat16", grad="bfloat16", drop=0.0, pad=0.0,
             alpha=1.05, scatter=True, rule="adagrad"),
    ]


def _log(rng, lo, hi):
    """A whole number spread over [lo, hi] by its logarithm (odd and ragged values come with it)."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["embed", "grad", "step"])
    dim = rng.choice([16, 24, 48, 50, 64, 100, 128, 200, 256, 333, 512, 1000, 1024]) if op == "step" else rng.choice(
        [16, 24, 48, 50, 64, 100, 128, 200, 256, 333, 512, 1000, 1024, 2048, 4096])
    table, grad = rng.choice(["float32", "bfloat16", "bfloat16", "float16"]), rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    most = 1_000_000 if op == "step" else 2_000_000
    n = _log(rng, 1, most)
    n = max(1, min(n, (128 * most) // dim))
    rows = max(1000, min(_log(rng, 1000, 25_000_000 if op != "step" else 6_000_000), 700_000_000 // dim))
    return dict(op=op, n=n, rows=rows, dim=dim, table=table, grad=grad, drop=rng.choice([0.0, 0.0, 0.1, 0.25, 0.5]),
                pad=rng.choice([0.0, 0.0, 0.05, 0.3]), alpha=round(rng.uniform(1.02, 1.2), 3), scatter=rng.choice([True, True, False]),
                rule=rng.choice(["adagrad", "adagrad", "sgd"]) if op == "step" else "")


def _ranks(u, alpha, universe):
    """Bounded Pareto ranks in [1, universe] of uniform numbers u, as in the streams of the training workloads."""
    one_m = 1.0 - alpha
    top = float(universe + 1) ** one_m
    return (((top - 1.0) * u + 1.0) ** (1.0 / one_m)).floor()


def _scale(case):
    return math.sqrt(case["dim"])                  # what a lookup in front of a transformer multiplies by


_kept = SimpleNamespace(handle=None)               # a program has one handle for the scratch of its gradients


def _handle(n, dim):
    from paper_2602_17050_amd import binding as mp
    if _kept.handle is None:
        _kept.handle = mp.mpzch_embed_create()
    mp.mpzch_embed_reserve(_kept.handle, n, dim)
    return _kept.handle


# ------------------------------------------------------------------------------------------------ inputs
def _slots(case, g):
    u = torch.rand(case["n"], generator=g, device=DEVICE, dtype=torch.float64)
    rank = _ranks(u, case["alpha"], case["rows"]).clamp_(max=case["rows"]).to(torch.int64) - 1
    if case["scatter"]:                            # a table's slots: the hash has spread the ids
        start = int(torch.randint(1 << 40, (1,), generator=g, device=DEVICE).item())
        rank = (((rank + start) * (GOLDEN - (1 << 64))) >> 8) & ((1 << 52) - 1)
        rank = rank % case["rows"]
    if case["pad"]:
        rank[torch.rand(case["n"], generator=g, device=DEVICE) < case["pad"]] = -1
    return rank


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    s = SimpleNamespace(case=case, op=case["op"], n=case["n"], num_rows=case["rows"], dim=case["dim"], drop=case["drop"],
                        scale=_scale(case), handle=None)
    s.slots = _slots(case, g)
    s.seed = torch.randint(-(1 << 62), 1 << 62, (1,), generator=g, device=DEVICE, dtype=torch.int64)
    wide, narrow = DTYPES[case["table"]], DTYPES[case["grad"]]
    if case["op"] != "embed":
        s.grad = (torch.randn(s.n, s.dim, generator=g, device=DEVICE) * 0.01).to(narrow)
    if case["op"] != "grad":
        s.rows = torch.empty(s.num_rows, s.dim, dtype=wide, device=DEVICE).normal_(0.0, 1.0 / math.sqrt(s.dim), generator=g)
    if case["op"] == "embed":
        s.out = torch.empty(s.n, s.dim, dtype=narrow, device=DEVICE)
    elif case["op"] == "grad":
        s.out_slots = torch.zeros(s.n, dtype=torch.int64, device=DEVICE)
        s.out_rows = torch.zeros(s.n, s.dim, dtype=wide, device=DEVICE)
        s.count = torch.zeros(1, dtype=torch.int64, device=DEVICE)
    else:
        s.state = torch.rand(s.num_rows, generator=g, device=DEVICE) * 0.1 if case["rule"] == "adagrad" else None
        s.lr = torch.full((1,), LR, device=DEVICE)
    if own and case["op"] != "embed":
        s.handle = _handle(s.n, s.dim)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _threshold(drop):
    return int(math.floor(drop * 65536 + 0.5))


def _signed(v):
    return v - (1 << 64) if v >= 1 << 63 else v


def _shifted(z, k):
    return (z >> k) & ((1 << (64 - k)) - 1)        # torch has no unsigned shift


def _factor(s):
    return s.scale * 65536 / (65536 - _threshold(s.drop))


def _keep(s):
    """The truth values of the mask, n x dim; None without dropout."""
    t = _threshold(s.drop)
    if t == 0:
        return None
    words = (s.dim + 3) // 4
    z = torch.arange(1, s.n * words + 1, device=DEVICE) * _signed(GOLDEN) + s.seed
    z = (z ^ _shifted(z, 30)) * _signed(MIX[0])
    z = (z ^ _shifted(z, 27)) * _signed(MIX[1])
    z = z ^ _shifted(z, 31)
    draws = (z[:, None] >> torch.arange(0, 64, 16, device=DEVICE)) & 0xFFFF
    return (draws >= t).view(s.n, 4 * words)[:, : s.dim]


def _sums(s):
    """The rows that are named, ascending, and the sum for each: running sums over the sorted positions, in 64 bits since they
    run over the whole batch, and their differences from run to run."""
    order = torch.argsort(s.slots, stable=True)
    order = order[s.slots[order] >= 0]
    rows, lengths = torch.unique_consecutive(s.slots[order] % s.num_rows, return_counts=True)
    g = s.grad.float()
    keep = _keep(s)
    if keep is not None:
        g = torch.where(keep, g, 0.0)
    ends = g[order].double().t().contiguous().cumsum(1)[:, lengths.cumsum(0) - 1]       # (torch's scan of rows is the fast one)
    total = torch.diff(ends, dim=1, prepend=torch.zeros_like(ends[:, :1])).t()
    return rows, (total * _factor(s)).float()


def run(s):
    if own:
        from paper_2602_17050_amd import binding as mp
        if s.op == "embed":
            mp.mpzch_embed(s.slots, s.rows, s.out, scale=s.scale, drop_p=s.drop, seed=s.seed)
            return {"out": s.out}
        if s.op == "grad":
            mp.mpzch_embed_grad(s.handle, s.slots, s.grad, s.num_rows, s.out_slots, s.out_rows, s.count, scale=s.scale,
                                drop_p=s.drop, seed=s.seed)
            return {"slots": s.out_slots, "rows": s.out_rows, "count": s.count}
        mp.mpzch_embed_step(s.handle, s.slots, s.grad, s.rows, s.state, s.lr, EPS, scale=s.scale, drop_p=s.drop, seed=s.seed)
        return {"rows": s.rows, "state": s.state}
    if s.op == "embed":
        x = s.rows[s.slots.clamp(min=0) % s.num_rows].float() * _factor(s)
        x = torch.where((s.slots >= 0)[:, None], x, 0.0)
        keep = _keep(s)
        if keep is not None:
            x = torch.where(keep, x, 0.0)
        return {"out": x.to(s.out.dtype)}
    rows, total = _sums(s)
    if s.op == "grad":
        u = rows.numel()
        s.out_slots[:u] = rows
        s.out_rows[:u] = total.to(s.out_rows.dtype)
        s.count.fill_(u)
        return {"slots": s.out_slots, "rows": s.out_rows, "count": s.count}
    if s.state is None:
        s.rows[rows] = (s.rows[rows].float() - s.lr * total).to(s.rows.dtype)
    else:
        state = s.state[rows] + (total * total).mean(1)
        s.state[rows] = state
        s.rows[rows] = (s.rows[rows].float() - s.lr * (total / (state.sqrt() + EPS)[:, None])).to(s.rows.dtype)
    return {"rows": s.rows, "state": s.state}


# ------------------------------------------------------------------------------------------------ from the definition, 64 bits
def _mask64(case, seed_value):
    """numpy's unsigned words, by blocks of rows; truth values n x dim, or None."""
    t = int(case["drop"] * 65536 + 0.5)
    if not t:
        return None, 1.0
    words = -(-case["dim"] // 4)
    mask = np.empty((case["n"], case["dim"]), dtype=bool)
    some = max(1, (1 << 24) // words)
    with np.errstate(over="ignore"):
        for at in range(0, case["n"], some):
            m = min(some, case["n"] - at)
            x = np.arange(at * words, (at + m) * words, dtype=np.uint64)
            x = np.uint64(seed_value % (1 << 64)) + (x + np.uint64(1)) * np.uint64(GOLDEN)
            for shift, factor in ((30, MIX[0]), (27, MIX[1])):
                x ^= x >> np.uint64(shift)
                x *= np.uint64(factor)
            x ^= x >> np.uint64(31)
            draws = x.astype("<u8").view("<u2").reshape(m, 4 * words)
            mask[at:at + m] = draws[:, : case["dim"]] >= t
    return mask, 65536.0 / (65536.0 - t)


def exact(case, seed):
    s = prepare(case, seed)
    slots = s.slots.cpu().numpy()
    mask, grown = _mask64(case, int(s.seed.item()))
    f = math.sqrt(case["dim"]) * grown
    if case["op"] == "embed":
        there = np.flatnonzero(slots >= 0)
        out = np.zeros((case["n"], case["dim"]))
        out[there] = s.rows[torch.from_numpy(slots[there]).to(DEVICE)].double().cpu().numpy() * f
        if mask is not None:
            out[~mask] = 0.0
        return {"out": out}
    order = np.argsort(slots, kind="stable")
    order = order[np.searchsorted(slots[order], 0):]
    sorted_slots = slots[order]
    first = np.flatnonzero(np.concatenate([[True], sorted_slots[1:] != sorted_slots[:-1]])) if order.size else np.empty(0, np.int64)
    named = sorted_slots[first]
    total = np.zeros((named.size, case["dim"]))
    if order.size:
        g = s.grad.double().cpu().numpy()
        if mask is not None:
            g[~mask] = 0.0
        total = np.add.reduceat(g[order], first, axis=0) * f
    if case["op"] == "grad":
        out_slots, out_rows = np.zeros(case["n"], np.int64), np.zeros((case["n"], case["dim"]))
        out_slots[: named.size], out_rows[: named.size] = named, total
        return {"slots": out_slots, "rows": out_rows, "count": np.array([named.size])}
    at = torch.from_numpy(named).to(DEVICE)
    total = torch.from_numpy(total).to(DEVICE)
    rows, lr = s.rows.double(), float(s.lr.item())
    if case["rule"] == "sgd":
        rows[at] -= lr * total
        return {"rows": rows, "state": None}
    state = s.state.double()
    state[at] += total.square().sum(1) / case["dim"]
    rows[at] -= lr * total / (state[at].sqrt() + EPS)[:, None]
    return {"rows": rows, "state": state}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    n, dim, table, grad = case["n"], case["dim"], BYTES[case["table"]], BYTES[case["grad"]]
    g = torch.Generator()
    g.manual_seed(1)
    rank = _ranks(torch.rand(n, generator=g, dtype=torch.float64), case["alpha"], case["rows"])
    rank = rank[torch.rand(n, generator=g) >= case["pad"]]
    there, distinct = rank.numel(), torch.unique(rank).numel()
    if case["op"] == "embed":
        return {"bytes": 8 * n + distinct * dim * table + n * dim * grad, "flops": there * dim}
    read = 8 * n + there * dim * grad
    if case["op"] == "grad":
        return {"bytes": read + distinct * (8 + dim * table), "flops": there * dim}
    return {"bytes": read + 2 * distinct * dim * table + (8 * distinct if case["rule"] == "adagrad" else 0),
            "flops": (there + 4 * distinct) * dim}
