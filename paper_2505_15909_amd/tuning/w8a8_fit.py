#!/usr/bin/env python3
"""Fits the W8A8 product's model of its launches' time to sweeps (w8a8_sweep), and says how far the picks are behind.

  python paper_2505_15909_amd/tuning/w8a8_fit.py SWEEP [SWEEP ...] [--held-out SWEEP ...]
  python paper_2505_15909_amd/tuning/w8a8_fit.py --picks SWEEP ...           (the library's own picks, marked in the sweeps)
  python paper_2505_15909_amd/tuning/w8a8_fit.py --shorten SWEEP ...         (the launches within 1.6 times the fastest)

A fit prints the constants as csrc/rtn_w8a8_plan.h has them, and for the launches that the fitted model picks the time over that of the fastest launch, as
the logarithm of that ratio: mean and 95th percentile by rows, and the worst.  The model is the header's, its comment says what it is made of.
w8a8_sweep_results.txt holds the shortened sweeps that the header's constants are fitted to, w8a8_sweep_heldout.txt those of another card and other problems.
"""
import math
import os
import re
import sys

import numpy as np
import torch

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "csrc", "rtn_w8a8_plan.h")
STREAM, BLOCK, TILE = range(3)
SHAPES = [(["STREAM", "BLOCK", "TILE"].index(m[0]),) + tuple(map(int, m[1:5])) + tuple(map(float, m[5:8]))
          for m in re.findall(r"\{W8A8_(\w+), (\d+), (\d+), (\d+), (\d+), ([\d.]+)f, ([\d.]+)f, ([\d.]+)f\}", open(HEADER).read())]
COUNT = len(SHAPES)
KIND, DEPTH = np.array([s[0] for s in SHAPES]), np.array([max(s[4], 1) for s in SHAPES])
LAYERS = {(6144, 4096), (4096, 4096), (28672, 4096), (4096, 14336), (10240, 8192), (8192, 8192), (57344, 8192), (8192, 28672), (18432, 16384), (16384, 16384),
          (106496, 16384), (16384, 53248), (5120, 5120)}     # matrices of layers count more
MOST_TILES = 128                                             # of 128 rows x 256 columns, where block kernels are considered for more than 128 rows
LAYER_WEIGHT = 8.0
BANDS = [(1, 1), (2, 16), (17, 40), (41, 128), (129, 512), (513, 1024), (1025, 2048), (2049, 4096), (4097, 8192)]


def up(a, b):
    return -(-a // b)


def read(paths):
    """[(M, N, K), {(shape, split): us}, own pick]"""
    problems = []
    for path in paths:
        for line in open(path):
            if line.startswith("#"):
                continue
            head, *cells = line.strip().split(" | ")
            times, own = {}, None
            for cell in cells:
                shape, split, us, star = re.match(r"(\d+)/(\d+) ([\d.]+)(\*?)", cell).groups()
                times[int(shape), int(split)] = float(us)
                own = (int(shape), int(split)) if star else own
            problems.append((tuple(map(int, head.split())), times, own))
    return problems


def features(p, shape, split):
    """Workgroups along N and M, steps of a workgroup, workgroups on the fullest compute unit (a fraction), share of its rows that M has."""
    M, N, K = p
    kind, mb, nt, wk = SHAPES[shape][:4]
    if kind == TILE:
        XB, YB, steps, rows = up(N, 256), up(M, 32 * mb), 2 * up(K // 256, split), 32 * mb
    elif kind == BLOCK:
        XB, YB, steps, rows = up(N, 128 * nt // wk), up(M, 16 * mb), up(up(K // 128, split), wk), 16 * mb
    else:
        XB, YB, steps, rows = up(N, 16 * nt), up(M, 16 * mb), up(up(K // 64, split), wk), 16 * mb
    return XB, YB, steps, XB * YB * split / 256 if kind == STREAM else up(XB * YB, 8) * split / 32, M / (YB * rows)


def considered(p, shape):
    M, N, _ = p
    kind, mb = SHAPES[shape][:2]
    if kind == STREAM:
        return up(M, 16 * mb) <= 8
    return kind == TILE or M <= 128 or up(M, 128) * up(N, 256) <= MOST_TILES


def table(problems):
    cells = [(j, i, s, t, min(times.values())) + p + features(p, i, s) for j, (p, times, _) in enumerate(problems) for (i, s), t in times.items() if considered(p, i)]
    names = ("problem", "shape", "split", "us", "best", "M", "N", "K", "XB", "YB", "steps", "full", "rows")
    d = {n: np.array(c, float) for n, c in zip(names, zip(*cells))}
    return {n: torch.tensor(v.astype(int) if n in ("problem", "shape") else v) for n, v in d.items()}


NAMES = ("stream_rate", "join", "join_rate", "out_rate", "tile_round", "shared_stream", "shared_near", "shared_far", "join_tile", "tile_alone", "block_round")
IN_HEADER = ("kStreamRate", "kJoin", "kJoinRate", "kOutRate", "kTileRound", "kSharedStream", "kSharedNear", "kSharedFar", "kJoinTile", "kTileAlone", "kBlockRound")


def model(x, d):
    start, (each, more), g = x[0], x[1:3].exp(), dict(zip(NAMES, x[3].exp()))
    i, steps, full = d["shape"], d["steps"], d["full"]
    kind, none, one = torch.tensor(KIND)[i], torch.zeros_like(full), torch.ones_like(full)
    tile, size = kind == TILE, d["N"] * d["K"]
    shared = torch.where(kind == STREAM, g["shared_stream"], torch.where(size <= 32 << 20, g["shared_near"], g["shared_far"]))
    many = torch.ceil(full)
    work = steps * many * (each[i] + more[i] * d["rows"]) * torch.where(d["YB"] > 1, shared, one)
    work = work + torch.where(kind == BLOCK, g["block_round"] * (torch.ceil(many / torch.tensor(DEPTH)[i]) - 1), none)
    whole, part = torch.floor(full), full - torch.floor(full)
    tiles = steps * (whole * (each[i] + more[i]) + torch.where(part > 0, each[i] + more[i] * torch.clamp(2 * part - 1, min=0), none)) + g["tile_round"] * (whole + (part > 0) - 1)
    work = torch.where(tile, tiles * torch.where(d["YB"] == 1, g["tile_alone"], one), work)
    stream, out = (size + d["M"] * d["K"]) / g["stream_rate"] / 1e6, 2 * d["M"] * d["N"]
    t = start[i] + (work ** 4 + stream ** 4) ** 0.25 + torch.where(tile, none, out / g["out_rate"] / 1e6)
    return t + torch.where(d["split"] > 1, torch.where(tile, g["join_tile"], g["join"]) + out * (1 + 4 * d["split"]) / g["join_rate"] / 1e6, none)


def behind(problems, picks, worst=8):
    g = [(math.log(times[pick] / min(times.values())), p, pick, times[pick], min((t, c) for c, t in times.items())) for (p, times, _), pick in zip(problems, picks)]
    for lo, hi in BANDS:
        v = sorted(x[0] for x in g if lo <= x[1][0] <= hi)
        if v:
            print(f"  {lo:5d} to {hi:5d} rows: {len(v):4d} problems, mean {sum(v) / len(v):.3f}, 95 % {v[int(0.95 * len(v))]:.3f}, most {v[-1]:.3f}")
    print(f"  all: {len(g)} problems, mean {sum(x[0] for x in g) / len(g):.4f}")
    for x in sorted(g, reverse=True)[:worst]:
        print("    %.3f  %d rows of %d x %d: %d/%d %.1f us, best %d/%d %.1f" % (x[0], *x[1], *x[2], x[3], *x[4][1], x[4][0]))


def model_picks(x, problems):
    d = table(problems)
    best = {}
    for j, i, s, t in zip(d["problem"].tolist(), d["shape"].tolist(), d["split"].tolist(), model(x, d).tolist()):
        if j not in best or t < best[j][0]:
            best[j] = (t, (i, int(s)))
    return [best[j][1] for j in range(len(problems))]


def fit(paths, held_out, turns=600, nearness=0.03, times_share=0.3):
    """Descends from the header's constants on the mean of what a pick costs: the launches' logarithms over the fastest's, each by exp(-log(its modelled
    time) / nearness), a smooth stand-in for the least.  A share of the difference between modelled and measured times keeps the constants times."""
    problems = read(paths)
    d = table(problems)
    text = open(HEADER).read()
    value = [float(re.search(n + r" = ([\d.]+)(e6)?f", text)[1]) for n in IN_HEADER]
    log = lambda v: math.log(max(v, 0.004))                                             # noqa: E731
    width = max(COUNT, len(NAMES))
    x = torch.tensor([[s[5] for s in SHAPES], [log(s[6]) for s in SHAPES], [log(s[7]) for s in SHAPES], [log(v) for v in value] + [0.0] * (width - len(NAMES))],
                     dtype=torch.float64).requires_grad_(True)
    n, behind_best, near = len(problems), torch.log(d["us"] / d["best"]), (d["best"] / d["us"]) ** 3 * (d["us"] < 2.5 * d["best"])
    counts = torch.tensor([LAYER_WEIGHT if p[1:] in LAYERS else 1.0 for p, *_ in problems], dtype=torch.float64)
    optimizer = torch.optim.Adam([x], lr=0.004)
    for turn in range(turns):
        t = torch.log(model(x, d).clamp(min=0.1))
        chance = -t / (nearness * (1 - 0.6 * turn / turns))
        most = torch.full((n,), -1e30, dtype=torch.float64).scatter_reduce(0, d["problem"], chance.detach(), "amax")
        chance = torch.exp(chance - most[d["problem"]])
        total = torch.zeros(n, dtype=torch.float64)
        cost = total.scatter_add(0, d["problem"], chance * behind_best) / total.scatter_add(0, d["problem"], chance)
        off = ((t - torch.log(d["us"])) * near)[near > 0]
        loss = (cost * counts).sum() / counts.sum() + times_share * torch.nn.functional.huber_loss(off, torch.zeros_like(off), delta=0.2)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
    x = x.detach()
    off = torch.log(d["us"] / model(x, d)) ** 2
    for i, s in enumerate(SHAPES):
        of = d["shape"] == i
        rms = math.sqrt((off * near)[of].sum() / near[of].sum())
        print("    {W8A8_%s, %d, %d, %d, %d, %.3ff, %.3ff, %.3ff},   %d launches, rms %.2f" %
              (("STREAM", "BLOCK", "TILE")[s[0]], *s[1:5], x[0, i], x[1, i].exp(), x[2, i].exp(), of.sum(), rms))
    for name, v in zip(NAMES, x[3].exp()):
        print(f"    {name} {v:.3f}")
    print(f"{len(d['us'])} launches")
    behind(problems, model_picks(x, problems))
    if held_out:
        print("held out:")
        behind(read(held_out), model_picks(x, read(held_out)))


def main(args):
    if args[0] == "--picks":
        problems = read(args[1:])
        behind(problems, [own for *_, own in problems], 25)
    elif args[0] == "--shorten":
        print("# M N K | shape/split us | ... up to 1.6 times the fastest, * the library's pick at the time (w8a8_sweep)")
        for (M, N, K), times, own in read(args[1:]):
            print(f"{M} {N} {K}" + "".join(f" | {i}/{s} {round(t, 2 if t < 10 else 1 if t < 100 else 0):g}" + ("*" if (i, s) == own else "") for (i, s), t in times.items() if t <= 1.6 * min(times.values()) or (i, s) == own))
    else:
        at = args.index("--held-out") if "--held-out" in args else len(args)
        fit(args[:at], args[at + 1:])


if __name__ == "__main__":
    main(sys.argv[1:])
