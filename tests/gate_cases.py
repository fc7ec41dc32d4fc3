"""The gate's definition over whole batches in 64 bits (torch, on any device), inputs at which a choice can go wrong, and a pair of cases for each form
of its kernel."""
import itertools

import numpy as np
import torch

MASKED = float(np.float32(-1e30))
LARGEST = float(np.finfo(np.float32).max)
MASKS = ("none", "wild", "ties", "near", "pairs", "alike")

# (keys of a list, lanes of a token, experts of a lane, all lanes full): two cases (T, E, k, groups) that run it, the second with as many choices as keys
FORMS = {
    (4, 8, 8, 0): ((4101, 26, 3, 2), (4101, 59, 4, 1)), (4, 8, 8, 1): ((4101, 48, 3, 3), (4101, 64, 4, 2)),
    (4, 8, 16, 0): ((4101, 116, 3, 4), (4101, 125, 4, 1)), (4, 8, 16, 1): ((4101, 80, 1, 5), (4101, 128, 4, 1)),
    (4, 8, 24, 0): ((4101, 180, 1, 4), (4101, 147, 4, 1)), (4, 8, 24, 1): ((4101, 192, 3, 4), (4101, 168, 4, 7)),
    (4, 8, 32, 0): ((4101, 194, 3, 2), (4101, 238, 4, 2)), (4, 8, 32, 1): ((4101, 256, 2, 4), (4101, 256, 4, 8)),
    (4, 16, 8, 0): ((2053, 72, 3, 4), (2053, 104, 4, 8)), (4, 16, 8, 1): ((2053, 88, 1, 11), (2053, 104, 4, 13)),
    (4, 16, 16, 0): ((2053, 228, 3, 2), (2053, 140, 4, 1)), (4, 16, 16, 1): ((2053, 256, 1, 2), (2053, 256, 4, 2)),
    (4, 16, 24, 0): ((2053, 171, 1, 9), (2053, 370, 4, 1)), (4, 16, 24, 1): ((2053, 240, 3, 5), (2053, 288, 4, 6)),
    (4, 16, 32, 0): ((2053, 468, 2, 2), (2053, 286, 4, 11)), (4, 16, 32, 1): ((2053, 384, 3, 12), (2053, 288, 4, 9)),
    (4, 32, 8, 0): ((1029, 150, 3, 10), (1029, 160, 4, 16)), (4, 32, 8, 1): ((1029, 248, 3, 31), (1029, 240, 4, 30)),
    (4, 32, 16, 0): ((1029, 405, 3, 27), (1029, 481, 4, 1)), (4, 32, 16, 1): ((1029, 432, 1, 27), (1029, 496, 4, 31)),
    (4, 32, 24, 0): ((1029, 660, 1, 4), (1029, 744, 4, 4)), (4, 32, 24, 1): ((1029, 720, 3, 30), (1029, 768, 4, 4)),
    (4, 32, 32, 0): ((1029, 590, 3, 5), (1029, 800, 4, 8)), (4, 32, 32, 1): ((1029, 640, 1, 5), (1029, 576, 4, 18)),
    (4, 64, 8, 0): ((203, 216, 3, 6), (203, 472, 4, 8)), (4, 64, 8, 1): ((203, 344, 3, 43), (203, 400, 4, 50)),
    (4, 64, 16, 0): ((203, 805, 1, 7), (203, 845, 4, 1)), (4, 64, 16, 1): ((203, 976, 3, 61), (203, 848, 4, 53)),
    (4, 64, 24, 0): ((203, 843, 3, 3), (203, 966, 4, 23)), (4, 64, 24, 1): ((203, 1008, 3, 42), (203, 960, 4, 10)),
    (4, 64, 32, 0): ((203, 986, 2, 17), (203, 995, 4, 5)),
    (8, 8, 8, 0): ((4101, 35, 7, 7), (4101, 47, 8, 1)), (8, 8, 8, 1): ((4101, 64, 5, 8), (4101, 56, 8, 7)),
    (8, 8, 16, 0): ((4101, 93, 7, 3), (4101, 60, 8, 3)), (8, 8, 16, 1): ((4101, 128, 6, 1), (4101, 96, 8, 6)),
    (8, 8, 24, 0): ((4101, 154, 6, 2), (4101, 184, 8, 2)), (8, 8, 24, 1): ((4101, 192, 5, 8), (4101, 144, 8, 3)),
    (8, 8, 32, 0): ((4101, 198, 5, 2), (4101, 252, 8, 2)), (8, 8, 32, 1): ((4101, 192, 7, 6), (4101, 256, 8, 8)),
    (8, 16, 8, 0): ((2053, 39, 5, 13), (2053, 30, 8, 15)), (8, 16, 8, 1): ((2053, 120, 5, 15), (2053, 128, 8, 16)),
    (8, 16, 16, 0): ((2053, 120, 5, 3), (2053, 170, 8, 1)), (8, 16, 16, 1): ((2053, 160, 7, 5), (2053, 256, 8, 4)),
    (8, 16, 24, 0): ((2053, 228, 7, 12), (2053, 339, 8, 1)), (8, 16, 24, 1): ((2053, 288, 5, 12), (2053, 384, 8, 4)),
    (8, 16, 32, 0): ((2053, 416, 6, 2), (2053, 333, 8, 3)), (8, 16, 32, 1): ((2053, 288, 7, 9), (2053, 320, 8, 5)),
    (8, 32, 8, 0): ((1029, 180, 6, 30), (1029, 202, 8, 1)), (8, 32, 8, 1): ((1029, 248, 5, 31), (1029, 224, 8, 28)),
    (8, 32, 16, 0): ((1029, 348, 5, 6), (1029, 296, 8, 8)), (8, 32, 16, 1): ((1029, 448, 7, 28), (1029, 400, 8, 25)),
    (8, 32, 24, 0): ((1029, 350, 7, 10), (1029, 539, 8, 1)), (8, 32, 24, 1): ((1029, 408, 5, 17), (1029, 480, 8, 5)),
    (8, 32, 32, 0): ((1029, 572, 6, 11), (1029, 900, 8, 1)), (8, 32, 32, 1): ((1029, 928, 7, 29), (1029, 576, 8, 18)),
    (8, 64, 8, 0): ((203, 250, 7, 5), (203, 399, 8, 7)), (8, 64, 8, 1): ((203, 368, 6, 46), (203, 400, 8, 50)),
    (8, 64, 16, 0): ((203, 532, 7, 14), (203, 780, 8, 1)), (8, 64, 16, 1): ((203, 560, 7, 35), (203, 896, 8, 14)),
    (8, 64, 24, 0): ((203, 803, 5, 11), (203, 888, 8, 6)), (8, 64, 24, 1): ((203, 816, 6, 34), (203, 960, 8, 10)),
    (8, 64, 32, 0): ((203, 990, 5, 9), (203, 985, 8, 5)),
    (16, 16, 16, 0): ((2053, 162, 9, 6), (2053, 132, 16, 11)), (16, 16, 16, 1): ((2053, 256, 12, 8), (2053, 176, 16, 11)),
    (16, 16, 32, 0): ((2053, 435, 12, 15), (2053, 399, 16, 7)), (16, 16, 32, 1): ((2053, 384, 11, 6), (2053, 512, 16, 4)),
    (16, 32, 16, 0): ((1029, 280, 12, 2), (1029, 494, 16, 1)), (16, 32, 16, 1): ((1029, 384, 10, 6), (1029, 512, 16, 2)),
    (16, 32, 32, 0): ((1029, 540, 12, 5), (1029, 729, 16, 1)), (16, 32, 32, 1): ((1029, 768, 9, 6), (1029, 896, 16, 28)),
    (16, 64, 16, 0): ((203, 64, 9, 64), (203, 790, 16, 1)), (16, 64, 16, 1): ((203, 944, 12, 59), (203, 864, 16, 54)),
    (16, 64, 32, 0): ((203, 646, 12, 19), (203, 885, 16, 5)),
    # the general kernel: as many choices as groups of 64 experts have lanes, and more groups than a wavefront has
    (0, 64, 1, 0): ((203, 64, 17, 1), (203, 63, 63, 3)), (0, 64, 2, 0): ((203, 100, 4, 100), (203, 128, 100, 2)),
    (0, 64, 4, 0): ((203, 256, 17, 8), (203, 201, 64, 67)), (0, 64, 8, 0): ((203, 512, 33, 128), (203, 500, 200, 1)),
    (0, 64, 16, 0): ((203, 1024, 20, 512), (203, 1000, 300, 4)),
}


def groups_of(case):
    """(groups kept, scores of a group's) of a case: half of the groups, or as many as have its choices; two where there are two."""
    T, E, k, groups = case
    size = E // groups
    return max(-(-groups // 2), -(-k // size)), min(2, size)


def make(case, mask, scores, seed=0):
    """logits [T, E], bias [E] fp32."""
    T, E = case[:2]
    rng = np.random.default_rng([seed, T, E, MASKS.index(mask)])
    logits = (rng.normal(size=(T, E)) + 0.5 * rng.normal(size=E)).astype(np.float32)
    bias = (0.05 * rng.normal(size=E)).astype(np.float32)
    if mask == "wild":   # whatever a mask may be made of, in places drawn
        for v in (-np.inf, np.nan, -1e30, -LARGEST, np.inf, LARGEST, -0.0, 0.0, -200.0):
            logits[rng.random((T, E)) < 0.08] = v
        logits[::5] = -np.inf
        bias[rng.random(E) < 0.05] = -np.inf
        bias[rng.random(E) < 0.05] = np.nan
    elif mask == "ties":
        logits = rng.choice(np.array([-1.0, 0.0, 0.5, 0.5, 1.0], np.float32), size=(T, E))
        bias = rng.choice(np.array([0.0, 0.0, 0.25], np.float32), size=E)
    elif mask == "alike":
        logits[:], bias[:] = 0.0, 0.0
    elif mask in ("near", "pairs"):   # scores plus bias that fp32 cannot tell apart: all of them, or two by two
        l = logits[0].astype(np.float64)
        s = 1 / (1 + np.exp(-l)) if scores == "sigmoid" else np.exp(l - l.max()) / np.exp(l - l.max()).sum()
        level = rng.permutation(E) // 2 / E if mask == "pairs" else 0.0
        bias = (0.75 + level - s).astype(np.float32)
        logits = np.nextafter(logits[0], np.where(rng.random((T, E)) < 0.5, np.inf, -np.inf).astype(np.float32)).astype(np.float32)
    return logits, bias


def gate_fwd(logits, bias, k, scores, groups, kept, best, renorm=True, scale=1.0, stay=None):
    """topk_idx [T, k], topk_w [T, k], the groups' scores [T, groups] in 64 bits of fp32 logits [T, E] and bias [E] or None.  stay [T, groups]: the
    groups that stay, if they are given."""
    T, E = logits.shape
    inf = float("inf")
    l = logits.double()
    masked = ~(l > MASKED)
    l = torch.where(masked, 0.0, l.clamp(max=LARGEST))
    if scores == "sigmoid":
        s = 1 / (1 + torch.exp(-l))
    else:
        alive = torch.where(masked, -inf, l)
        top = alive.amax(1, keepdim=True)
        e = torch.exp(alive - torch.where(top > -inf, top, 0.0))
        z = e.sum(1, keepdim=True)
        s = e / torch.where(z > 0, z, 1.0)
    s = torch.where(masked, 0.0, s)
    c = l if bias is None else s + bias.double()
    dead = masked | ~(c > MASKED)
    of = s if bias is None and best == 2 else c
    part = torch.sort(torch.where(dead, -inf, of).view(T, groups, E // groups), dim=2, descending=True)[0][:, :, :best]
    rating = torch.where(part > -inf, part, 0.0).sum(2)
    rating = torch.where(part[:, :, 0] > -inf, rating, -inf)
    if stay is None:
        stay = torch.zeros(T, groups, dtype=torch.bool, device=l.device)
        stay.scatter_(1, torch.sort(rating, dim=1, descending=True, stable=True)[1][:, :kept], True)
    key = torch.where(dead, -1.7e308, c).masked_fill(~stay.repeat_interleave(E // groups, 1), -inf)
    idx = torch.sort(key, dim=1, descending=True, stable=True)[1][:, :k]
    none = torch.gather(masked, 1, idx)
    if not renorm:
        return idx, scale * torch.where(none, 0.0, torch.gather(s, 1, idx)), rating
    # over the largest chosen one: scores far below zero keep their ratios
    lk = torch.where(none, -inf, torch.gather(l, 1, idx))
    top = lk.amax(1, keepdim=True)
    top = torch.where(top > -inf, top, 0.0)
    if scores == "softmax":
        w = torch.exp(lk - top)
    else:
        top = top.clamp(max=0.0)
        w = torch.where(none, 0.0, 1 / (torch.exp(top - lk) + torch.exp(top)))
    z = w.sum(1, keepdim=True)
    return idx, scale * w / torch.where(z > 0, z, 1.0), rating


# Two evaluations of a group's score in 64 bits: the sum of the exponentials is off by up to 66 roundings of 2^-53 (22 and 40 additions in another order,
# the division), under 2^-46 of a score, two scores are at most 2 together, and the roundings of c and of the sum are less: 2^-44 in all.  Groups that are
# nearer to the cut than that (equal, but for the order in which scores and biases are added) may stay or not.
DOUBT = 2.0 ** -44


def choices_in_doubt(logits, bias, k, scores, groups, kept, best, rating):
    """Every choice of one token (logits [1, E], rating [1, groups]) that the doubt about its groups' scores leaves."""
    r = rating[0]
    cut = torch.sort(r, descending=True)[0]
    sure = [g for g in range(groups) if r[g] > cut[min(kept, groups - 1)] + DOUBT]
    maybe = [g for g in range(groups) if g not in sure and r[g] >= cut[kept - 1] - DOUBT]
    for more in itertools.combinations(maybe, kept - len(sure)):
        stay = torch.zeros(1, groups, dtype=torch.bool, device=r.device)
        stay[0, list(sure) + list(more)] = True
        yield gate_fwd(logits, bias, k, scores, groups, kept, best, stay=stay)[0][0]
