"""Plain references of the calls for drafted trees and beams: lists and numpy for what is whole, fp64 for what is not."""

from __future__ import annotations

import math

import numpy as np
import torch

DH = 128


def ways(parents, base):
    """For every node the nodes from its root to it, itself last; [] for what is no node."""
    got = []
    for i, p in enumerate(parents):
        if base < 0 or p < -1 or p >= i:
            got.append([])
        elif p == -1:
            got.append([i])
        else:
            got.append(got[p] + [i] if got[p] else [])
    return got


def plan(parents, base, n_sink=0, n_local=-1):
    """(positions, seen): seen[i] the nodes that node i sees."""
    positions, seen = [], []
    for way in ways(parents, base):
        depth = len(way) - 1
        positions.append(base + depth if way else -1)
        seen.append({x for j, x in enumerate(way) if n_local < 0 or depth - j <= n_local or base + j < n_sink})
    return positions, seen


def as_words(seen, words):
    out = np.zeros((len(seen), words), np.uint32)
    for i, nodes in enumerate(seen):
        for x in nodes:
            out[i, x // 32] |= np.uint32(1) << np.uint32(x % 32)
    return out.view(np.int32)


def accept(parents, base, tokens, choices, first):
    """(path, next) of one tree; `first` None: any root does."""
    way = ways(parents, base)
    path, at, want = [], -1, first
    while True:
        down = [i for i, p in enumerate(parents) if way[i] and p == at and (want is None or tokens[i] == want)]
        if not down:
            return path, -1 if want is None else want
        at = down[0]
        path.append(at)
        want = choices[at]


def random_parents(rng, n, *, roots=1, gone=0.0, chain=0.3):
    """n parents: -1 for the first `roots`, now and then a chain, some that are no nodes."""
    out = []
    for i in range(n):
        if i < roots:
            out.append(-1)
        elif rng.random() < gone:
            out.append(rng.choice([-2, i, i + 1, 2 ** 31 - 1, -2 ** 31]))
        else:
            out.append(i - 1 if rng.random() < chain else rng.randrange(i))
    return out


def reorder(table, parents, kv_len, page):
    """(new table, moves of every beam as (src, dst) pool rows) of one group; `table` a list of rows."""
    n = len(parents)
    parents = [p if 0 <= p < n else i for i, p in enumerate(parents)]
    keeper = {}
    for i, p in enumerate(parents):
        if parents[p] == p:
            keeper[p] = p
        else:
            keeper.setdefault(p, i)
    free = [p for p in range(n) if p not in keeper]
    full, rest = divmod(max(kv_len, 0), page)
    new, moves = [], []
    for i, p in enumerate(parents):
        d = p if keeper[p] == i else free.pop(0)
        new.append(table[p][:full] + table[d][full:])
        moves.append([(table[p][full] * page + t, table[d][full] * page + t) for t in range(rest)]
                     if d != p and full < len(table[p]) else [])
    return new, moves


def apply_moves(pages, moves, page):
    """The moves of a group, in order, on a pool [pages][page][...] or, with heads between, scales [pages][heads][page]."""
    for src, dst in moves:
        if pages.dim() == 3:
            pages[dst // page, :, dst % page] = pages[src // page, :, src % page].clone()
        else:
            pages[dst // page, dst % page] = pages[src // page, src % page].clone()


def best(logits, scores, n_best):
    """[(score, beam, token)] of one group in 64 bits: logits fp64 [beams][vocab], scores [beams]."""
    z = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    top = z.max(-1)
    rows = []
    for i in range(z.shape[0]):
        if np.isfinite(scores[i]) and np.isfinite(top[i]):
            rows.append(np.float64(scores[i]) + (z[i] - (top[i] + math.log(np.exp(z[i] - top[i]).sum()))))
        else:
            rows.append(np.full(z.shape[1], -np.inf))
    flat = np.concatenate(rows)
    order = np.argsort(-flat, kind="stable")[:n_best]
    return [(flat[x], int(x) // z.shape[1], int(x) % z.shape[1]) for x in order]


def attend_tree64(bt, q, seen, positions, n_sink=0, n_local=-1, scale=None):
    """(out, lse, bound of out, bound of lse) in fp64. seen[r]: the nodes that row r sees. The bounds are those of
    attend64 (products exact in fp32, 128 of them summed, two roundings and the exponential's 2^-21 on the
    way to a weight, a weight rounded to 8 bits, n sums in fp32, the output rounded to bf16)."""
    scale = 1 / math.sqrt(DH) if scale is None else scale
    g = bt.hq // bt.hkv
    outs, lses, tol_o, tol_l = [], [], [], []
    row = 0
    for b, (a, n) in enumerate(zip(bt.news, bt.lens)):
        if a == 0:
            continue
        base = n - a
        sees = torch.zeros(a, max(n, 0), dtype=torch.bool)
        for i in range(a):
            p = positions[row + i]
            if p < 0 or base + i < 0:
                continue
            p = max(p, base)
            if base > 0:
                sees[i, :base] = True
                if n_local >= 0:
                    sees[i, n_sink: max(n_sink, min(base, p - n_local))] = False
            for c in seen[row + i]:
                if c < a and base + c >= 0:
                    sees[i, base + c] = True
        sees = sees.cuda()
        k, v = (bt.values[x][b].repeat_interleave(g, 1).transpose(0, 1) for x in range(2))
        x = q[row: row + a].double().transpose(0, 1)
        z = torch.where(sees, x @ k.transpose(1, 2) * scale, -math.inf)
        size = torch.where(sees, x.abs() @ k.abs().transpose(1, 2) * abs(scale), 0.0)
        if n > 0:
            top, big = z.amax(-1, keepdim=True), size.amax(-1, keepdim=True)
            logit = z.abs().masked_fill(~sees, 0).amax(-1, keepdim=True)
        else:
            top = torch.full((bt.hq, a, 1), -math.inf, device="cuda", dtype=torch.float64)
            big = logit = torch.zeros_like(top)
        w = torch.exp(z - top.clamp(min=-1e300))
        total = w.sum(-1, keepdim=True)
        w = w / total.clamp(min=1e-300)
        out, spread = w @ v, w @ v.abs()
        delta = 2 * 128 * 2.0 ** -24 * big + 8 * 2.0 ** -24 * logit + 2.0 ** -21
        sums = 2 * max(n, 1) * 2.0 ** -24
        lse = (total.log() + top)[..., 0]
        outs.append(out.transpose(0, 1))
        lses.append(lse.t())
        tol_o.append((2.0 ** -8 * out.abs() + (2.0 ** -8 + 2 * delta + sums) * spread + 2.0 ** -130).transpose(0, 1))
        tol_l.append((delta + sums + 2.0 ** -22 * lse[..., None].abs().nan_to_num(posinf=0, neginf=0))[..., 0].t())
        row += a
    return tuple(torch.cat(x) for x in (outs, lses, tol_o, tol_l))
