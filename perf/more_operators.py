"""Performance cases of the paged cache: the write of rotated rows into pages,
attention of sequences that share pages, and the forks of such sequences.

Each case is one pass through one operator, as a user of ``paper_2608_19147_amd``
calls it (``own``), or its plain form in elementary torch operations.

* ``write``: new rows q | k | v; pair (i, i + D/2) of every q and k head turns by
  p[axis(i)] theta^(-2i/D), with one position per row (text) or three (time,
  height, width of an image's patches); k and v go to their rows of the pages, q
  comes back.  Outputs: q and the pages;
* ``attend``: o = sum_j w_j v_j / sum_j w_j, w_j = exp(q.k_j / sqrt(D)), over the
  rows j of its sequence that a new row sees: those up to its own, less what a mask
  hides.  All sequences begin with ``system`` rows, the sequences of each of
  ``groups`` groups go on with the same ``shared`` rows, then each has its own;
* ``fork``: new sequences that begin as others do: whole pages are shared, the rows
  of a last page that is not full are copied.  With ``drop``, a share of the rows is
  left out and the ones behind close up, in pages of the new sequence's own.
  Output: the pages.

A pool hands out its lowest-numbered free pages first.  Sizes are those of the
repository's shapes (32 or 64 query heads, 8 kv heads, heads of 64 or 128, half
stages of 16 layers, 64 rows a forward, prompts of 2048) and generic ones.
"""
from __future__ import annotations

import functools
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
THETA = 500000.0
POSITIONS = 16384


# ---------------------------------------------------------------------- cases

def listed():
    return [
        # one decoded token's row: the smallest call, all latency
        dict(name="write_token", kind="write", S=1, n=1, past=2047, Hq=32, Hkv=8, D=128, kv="bf16", x="bf16", page=64, axes=1, pad=0),
        # patches of three images behind a few words, positions on three axes, rows inside wider ones
        dict(name="write_image", kind="write", S=3, n=577, past=19, Hq=32, Hkv=8, D=128, kv="f16", x="f32", page=16, axes=3, pad=5),
        # two prompts' rows as a product leaves them, 32 bits each: bound by memory
        dict(name="write_prompt", kind="write", S=2, n=2048, past=0, Hq=64, Hkv=8, D=128, kv="bf16", x="f32", page=64, axes=1, pad=0),
        # one request, one token: nothing is shared, latency and the split of its rows count
        dict(name="attend_token", kind="attend", S=1, n=1, system=0, groups=1, shared=0, own=2048, Hq=32, Hkv=8, D=128, kv="bf16",
             page=64, mask="none"),
        # a full forward of decoding requests that began with one long prompt
        dict(name="attend_batch", kind="attend", S=64, n=1, system=0, groups=1, shared=4096, own=512, Hq=32, Hkv=8, D=128, kv="bf16",
             page=64, mask="none"),
        # drafted trees of two prompts' requests behind common instructions, rejected rows hidden, small heads, odd lengths
        dict(name="attend_tree", kind="attend", S=4, n=15, system=1001, groups=2, shared=2999, own=333, Hq=16, Hkv=4, D=64, kv="f16",
             page=16, mask="tree"),
        # long caches, nothing shared: bound by reading them
        dict(name="attend_long", kind="attend", S=4, n=1, system=0, groups=1, shared=0, own=131072, Hq=64, Hkv=8, D=128, kv="bf16",
             page=256, mask="none"),
        # verifies of five tokens, each request with hidden rows, on pages that end inside every tile
        dict(name="attend_verify", kind="attend", S=12, n=5, system=300, groups=3, shared=2048, own=777, Hq=64, Hkv=8, D=128, kv="bf16",
             page=32, mask="holes"),
        # prompts that go on from a common one: bound by the matrix cores
        dict(name="attend_prompt", kind="attend", S=4, n=1024, system=0, groups=1, shared=2048, own=1024, Hq=32, Hkv=8, D=128,
             kv="bf16", page=64, mask="none"),
        # one more answer to a short prompt: the smallest copy
        dict(name="fork_one", kind="fork", parents=1, children=1, rows=200, drop=0.0, L=16, Hkv=8, D=128, kv="bf16", page=64),
        # 64 answers to four prompts, each with its copy of the last rows
        dict(name="fork_batch", kind="fork", parents=4, children=16, rows=1000, drop=0.0, L=16, Hkv=8, D=128, kv="bf16", page=64),
        # conversations whose hidden rows go before they are kept
        dict(name="fork_compact", kind="fork", parents=4, children=1, rows=1201, drop=0.3, L=16, Hkv=8, D=128, kv="bf16", page=64),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("write", "write", "attend", "attend", "attend", "attend", "attend", "fork", "fork"))
    D, kv, page = rng.choice((64, 128, 128)), rng.choice(("bf16", "bf16", "f16")), rng.choice((16, 32, 64, 64, 128, 256))
    Hkv = rng.choice((1, 2, 4, 8, 8))
    Hq = min(64, Hkv * rng.choice((1, 2, 4, 4, 5, 7, 8, 16)))
    Hq = Hq // Hkv * Hkv
    if kind == "write":
        S = _log(rng, 1, 64)
        n = _log(rng, 1, max(1, 4096 // S))
        return dict(kind=kind, S=S, n=n, past=rng.randint(0, 2048), Hq=Hq, Hkv=Hkv, D=D, kv=kv, x=rng.choice((kv, "f32")), page=page,
                    axes=rng.choice((1, 3)), pad=rng.choice((0, 0, 3, 8)))
    if kind == "fork":
        c = dict(kind=kind, parents=rng.randint(1, 4), children=1, rows=_log(rng, 1, 1200), drop=rng.choice((0.02, 0.3, 0.7)),
                 L=rng.choice((1, 4, 16)), Hkv=Hkv, D=D, kv=kv, page=page)
        if rng.random() < 0.5:
            c.update(children=_log(rng, 1, 16), drop=0.0)
            c["rows"] += c["rows"] % page == 0                   # whole pages are shared without a copy
        return c
    form = rng.choice(("decode", "decode", "verify", "verify", "prompt", "long"))
    c = dict(kind=kind, S=_log(rng, 1, 64), n=1, system=0, groups=1, shared=0, own=_log(rng, 1, 2048), Hq=Hq, Hkv=Hkv, D=D, kv=kv,
             page=page, mask=rng.choice(("none", "none", "holes")))
    if form == "long":
        c.update(S=rng.randint(1, 4), own=_log(rng, 2048, 131072))
        return c
    if rng.random() < 0.7:
        c.update(shared=_log(rng, 16, 8192), groups=rng.randint(1, min(4, c["S"])), system=rng.choice((0, 0, _log(rng, 16, 2048))))
    if form == "verify":
        c.update(n=rng.randint(2, 16), S=min(16, c["S"]), mask=rng.choice(("none", "holes", "tree")))
    if form == "prompt":
        c.update(n=_log(rng, 17, 1024), S=min(4, c["S"]), shared=min(2048, c["shared"]), own=_log(rng, 1, 1024), Hq=min(Hq, 32) // Hkv * Hkv)
        c.update(system=min(256, c["system"]))
    c["groups"] = min(c["groups"], c["S"])
    c["own"] = max(c["own"], 2 * c["n"])                         # the shortest sequence's own rows hold its new ones
    return c


def _own_rows(case):
    """Own rows of each sequence, new ones included: ragged, from ``own`` down to about half of it."""
    S, own_ = case["S"], case["own"]
    return [max(case["n"], own_ - (i * own_) // (2 * S)) for i in range(S)]


def _group(case):
    return [i * case["groups"] // case["S"] for i in range(case["S"])]


# --------------------------------------------------------------------- inputs

def _gen(seed, at):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) & 0xFFFFFFFF) * 1000003 + at)
    return g


def _host(seed, at):
    return np.random.default_rng([int(seed) & 0xFFFFFFFF, at])


def _qkv(case, seed):
    """q [M, Hq D], k and v [M, Hkv D] as parts of one product's rows, and positions int32 [axes, M]."""
    S, n, D = case["S"], case["n"], case["D"]
    nq, nk = case["Hq"] * D, case["Hkv"] * D
    x = torch.randn((S * n, nq + 2 * nk + case["pad"]), device="cuda", generator=_gen(seed, 0)) * 1.5
    x[:, :: 61] *= 6.0                                           # a few large channels
    x = x.to(TORCH[case["x"]])
    t = np.tile(case["past"] + np.arange(n), S)
    if case["axes"] == 3:                                        # words, then patches row by row
        r = _host(seed, 1)
        wide, start = max(1, math.isqrt(n)), r.integers(0, 64, S).repeat(n)
        i = np.tile(np.arange(n), S)
        t = np.stack([case["past"] + start, case["past"] + start + i // wide, case["past"] + start + i % wide])
    return x[:, :nq], x[:, nq:nq + nk], x[:, nq + nk:nq + 2 * nk], t.reshape(case["axes"], S * n).astype(np.int32)


def _pair_axis(case):
    """The axis whose position turns pair i: all the first, or a quarter of the pairs time, the others height and width."""
    half = case["D"] // 2
    if case["axes"] == 1:
        return None
    hw = half * 3 // 8
    return np.array([0] * (half - 2 * hw) + [1] * hw + [2] * hw, np.uint8)


def _segments(case, seed):
    """K and V of the system rows [Hkv, P0, D], the groups' [G, Hkv, P1, D] and the sequences' own [S, Hkv, own, D], and q [M, Hq D]."""
    g, dt = _gen(seed, 2), TORCH[case["kv"]]
    Hkv, D = case["Hkv"], case["D"]

    def rows(*lead, n):
        k = torch.randn((*lead, Hkv, n, D), device="cuda", generator=g)
        k[..., ::37, :] *= 2.5                                   # now and then a key that draws much of the weight
        return k.to(dt), torch.randn((*lead, Hkv, n, D), device="cuda", generator=g).to(dt)

    seg = [rows(n=case["system"]), rows(case["groups"], n=case["shared"]), rows(case["S"], n=case["own"])]
    q = (torch.randn((case["S"] * case["n"], case["Hq"] * D), device="cuda", generator=g) * 1.2).to(dt)
    return seg, q


def _masks(case, seed):
    """Per sequence: a uint8 [T] mask of its rows or None, and uint8 [n, T] masks of its new rows or None."""
    r, n, out = _host(seed, 3), case["n"], []
    for own_ in _own_rows(case):
        T = case["system"] + case["shared"] + own_
        mask = rows = None
        if case["mask"] != "none":
            mask = (r.random(T) >= 0.06).astype(np.uint8)
            mask[T - n:] = 1
        if case["mask"] == "tree":
            rows = np.ones((n, T), np.uint8)
            rows[:, T - n:] = 0
            for i in range(n):
                rows[i, T - n + i] = 1
                if i:
                    p = int(r.integers(max(0, i - 4), i))
                    rows[i, T - n:] |= rows[p, T - n:]
        out.append((mask, rows))
    return out


def _keeps(case, seed):
    r = _host(seed, 4)
    return [(r.random(case["rows"]) >= case["drop"]).astype(np.uint8) for _ in range(case["parents"])]


def _parent_rows(case, seed):
    g, dt = _gen(seed, 5), TORCH[case["kv"]]
    shape = (case["L"], case["Hkv"], case["rows"], case["D"])
    return [tuple(torch.randn(shape, device="cuda", generator=g).to(dt) for _ in range(2)) for _ in range(case["parents"])]


def _ceil(a, b):
    return -(-a // b)


def _fork_pages(case, keeps):
    """(kept rows, leading pages shared) of each child, in order."""
    out = []
    for i in range(case["parents"] * case["children"]):
        keep = keeps[i // case["children"]]
        kept = int(keep.sum())
        first = case["rows"] if keep.all() else int(np.argmin(keep))   # the rows before the first one left out stay where they are
        out.append((kept, min(first, kept) // case["page"]))
    return out


@functools.lru_cache(maxsize=4)
def _stage(L, Hq, Hkv, D, kv):
    """The stage that the cache belongs to: a program has one, whatever it calls on it."""
    from paper_2608_19147_amd import Stage

    g = torch.Generator().manual_seed(0)
    H, F = 256, 688
    dims = {"wq": (Hq * D, H), "wk": (Hkv * D, H), "wv": (Hkv * D, H), "wo": (H, Hq * D), "wg": (F, H), "wu": (F, H), "wd": (H, F)}
    mats = {name: SimpleNamespace(q=torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8).numpy(),
                                  scales=np.full((n, -(-k // 128)), 0.002, np.float16), n=n, k=k)
            for name, (n, k) in dims.items()}
    shape = SimpleNamespace(n_layers=L, hidden=H, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, ffn=F, group_size=128, rms_eps=1e-5,
                            rope_theta=THETA, act_dtype=kv, kv_dtype=kv, max_positions=POSITIONS)
    norm = torch.ones(H, dtype=TORCH[kv])
    return Stage(shape, [SimpleNamespace(attn_norm=norm, ffn_norm=norm, mats=mats)] * L)


def _prepare_own(s, case, seed):
    from paper_2608_19147_amd import PagedRequest

    dt, page, Hkv, D = TORCH[case["kv"]], case["page"], case["Hkv"], case["D"]
    if s.kind == "write":
        S, n, past = case["S"], case["n"], case["past"]
        stage = _stage(1, case["Hq"], Hkv, D, case["kv"])
        s.pool = stage.new_pages(S * (_ceil(past + n, page) + 1), page, pair_axis=_pair_axis(case))
        rows = torch.zeros((1, Hkv, past, D), dtype=dt, device="cuda")
        s.seqs = [s.pool.new_sequence() for _ in range(S)]
        for q in s.seqs:
            if past:
                q.append(rows, rows)
        s.step = s.pool.new_step()
        s.step.plan([PagedRequest(q, n, positions=s.positions[:, i * n:(i + 1) * n]) for i, q in enumerate(s.seqs)])
    elif s.kind == "attend":
        S, n = case["S"], case["n"]
        stage = _stage(1, case["Hq"], Hkv, D, case["kv"])
        sys_, grp, mine = s.seg
        pages = sum(_ceil(r, page) + 1 for r in [case["system"]] + [case["shared"]] * case["groups"] + [r + page for r in _own_rows(case)])
        s.pool = stage.new_pages(pages, page)
        base = s.pool.new_sequence()
        if case["system"]:
            base.append(sys_[0][None], sys_[1][None])
        heads = s.pool.fork([base] * case["groups"])
        for g, h in enumerate(heads):
            if case["shared"]:
                h.append(grp[0][g][None], grp[1][g][None])
        s.seqs = s.pool.fork([heads[g] for g in _group(case)])
        new = [[], []]
        for i, (q, r) in enumerate(zip(s.seqs, _own_rows(case))):
            if r > n:
                q.append(mine[0][i, None, :, :r - n], mine[1][i, None, :, :r - n])
            for j in range(2):
                new[j].append(mine[j][i, :, r - n:r].transpose(0, 1).reshape(n, Hkv * D))
        s.kept = [base, *heads]
        s.step = s.pool.new_step()
        s.step.plan([PagedRequest(q, n, mask=m, mask_rows=r) for q, (m, r) in zip(s.seqs, s.masks)])
        s.step.write(0, s.q, torch.cat(new[0]), torch.cat(new[1]))
        s.seg = None
    else:
        stage = _stage(case["L"], Hkv, Hkv, D, case["kv"])
        s.pool = stage.new_pages(s.n_pages, page)
        s.parents = [s.pool.new_sequence() for _ in s.rows]
        for q, (k, v) in zip(s.parents, s.rows):
            q.append(k, v)
        s.rows = None


def _prepare_plain(s, case):
    dt, page, Hkv, D = TORCH[case["kv"]], case["page"], case["Hkv"], case["D"]
    if s.kind == "write":
        S, n, past = case["S"], case["n"], case["past"]
        head, all_ = _ceil(past, page), _ceil(past + n, page)
        row = past + np.arange(n)
        at = []                                                  # the past rows' pages of all sequences come first, then the new rows'
        for i in range(S):
            t = row // page
            at.append(np.where(t < head, i * head + t, S * head + i * (all_ - head) + t - head) * page + row % page)
        s.at = torch.from_numpy(np.concatenate(at)).cuda()
        s.positions = torch.from_numpy(s.positions).cuda()
        axis = _pair_axis(case)
        s.axis = torch.zeros(D // 2, dtype=torch.long, device="cuda") if axis is None else torch.from_numpy(axis.astype(np.int64)).cuda()
        shape = (1, S * (all_ + 1), Hkv, page, D)
        s.k_pages, s.v_pages = (torch.zeros(shape, dtype=dt, device="cuda") for _ in range(2))
    elif s.kind == "attend":
        S, n, own_ = case["S"], case["n"], _own_rows(case)
        past = case["system"] + case["shared"]
        see = torch.zeros((S, n, past + case["own"]), dtype=torch.bool, device="cuda")
        for i, (r, (mask, rows)) in enumerate(zip(own_, s.masks)):
            T = past + r
            m = torch.ones((n, T), dtype=torch.bool, device="cuda").tril(T - n)
            if mask is not None:
                m &= torch.from_numpy(mask).cuda().bool()
            if rows is not None:
                m &= torch.from_numpy(rows).cuda().bool()
            see[i, :, :T] = m
        s.see = see
        s.group = torch.tensor(_group(case), device="cuda")
    else:
        shape = (case["L"], s.n_pages, Hkv, page, D)
        s.k_pages, s.v_pages = (torch.zeros(shape, dtype=dt, device="cuda") for _ in range(2))
        per = _ceil(case["rows"], page)
        for i, rows in enumerate(s.rows):
            for p, r in zip((s.k_pages, s.v_pages), rows):
                r = torch.nn.functional.pad(r, (0, 0, 0, per * page - case["rows"]))
                p[:, i * per:(i + 1) * per] = r.view(case["L"], Hkv, per, page, D).transpose(1, 2)
        s.rows = None


def prepare(case, seed):
    s = SimpleNamespace(case=case, kind=case["kind"])
    if s.kind == "write":
        s.q, s.k, s.v, s.positions = _qkv(case, seed)
    elif s.kind == "attend":
        s.seg, s.q = _segments(case, seed)
        s.masks = _masks(case, seed)
    else:
        s.keeps, s.rows = _keeps(case, seed), _parent_rows(case, seed)
        s.n_pages = case["parents"] * (1 + case["children"]) * _ceil(case["rows"], case["page"]) if case["drop"] else \
            case["parents"] * (_ceil(case["rows"], case["page"]) + case["children"])
    if own:
        _prepare_own(s, case, seed)
    else:
        _prepare_plain(s, case)
    return s


# ----------------------------------------------------------------- plain form

def _turn(x, cos, sin):
    """[M, H, D] fp32 rows with pair (i, i + D/2) turned."""
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _plain_write(s, c):
    M, D, dt = s.q.shape[0], c["D"], TORCH[c["kv"]]
    i = torch.arange(D // 2, device="cuda", dtype=torch.float64)
    angle = s.positions.double()[s.axis].t() * torch.exp(-2.0 * i / D * math.log(THETA))   # [M, D/2]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _turn(s.q.float().reshape(M, c["Hq"], D), cos, sin).to(dt).view(M, -1)
    k = _turn(s.k.float().reshape(M, c["Hkv"], D), cos, sin).to(dt)
    v = s.v.float().reshape(M, c["Hkv"], D).to(dt)
    page = c["page"]
    s.k_pages[0, s.at // page, :, s.at % page] = k
    s.v_pages[0, s.at // page, :, s.at % page] = v
    return q, s.k_pages, s.v_pages


def _plain_attend(s, c):
    S, n, Hq, Hkv, D, G = c["S"], c["n"], c["Hq"], c["Hkv"], c["D"], c["groups"]
    gs, P0, P1 = Hq // Hkv, c["system"], c["shared"]
    q = s.q.float().view(S, n, Hkv, gs, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, gs * n, D) / math.sqrt(D)
    kv = [(k.float(), v.float()) for k, v in s.seg]
    scores = []
    all_q = q.transpose(0, 1).reshape(Hkv, S * gs * n, D)        # the rows of all sequences meet the common rows in one product
    scores.append((all_q @ kv[0][0].transpose(1, 2)).view(Hkv, S, gs * n, P0).transpose(0, 1))
    shared = torch.empty((S, Hkv, gs * n, P1), device="cuda")
    for g in range(G):
        at = (s.group == g).nonzero()[:, 0]
        qg = q[at].transpose(0, 1).reshape(Hkv, len(at) * gs * n, D)
        shared[at] = (qg @ kv[1][0][g].transpose(1, 2)).view(Hkv, len(at), gs * n, P1).transpose(0, 1)
    scores.append(shared)
    scores.append(q @ kv[2][0].transpose(2, 3))
    z = torch.cat(scores, -1).view(S, Hkv, gs, n, -1)
    z = z.masked_fill(~s.see[:, None, None], -torch.inf)
    top = z.amax(-1, keepdim=True)
    w = torch.exp(z - torch.where(top == -torch.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    w = (w / torch.where(total == 0, 1.0, total)).view(S, Hkv, gs * n, -1)
    w0, w1, w2 = w.split((P0, P1, c["own"]), -1)
    o = (w0.transpose(0, 1).reshape(Hkv, S * gs * n, P0) @ kv[0][1]).view(Hkv, S, gs * n, D).transpose(0, 1) + w2 @ kv[2][1]
    for g in range(G):
        at = (s.group == g).nonzero()[:, 0]
        og = w1[at].transpose(0, 1).reshape(Hkv, len(at) * gs * n, P1) @ kv[1][1][g]
        o[at] += og.view(Hkv, len(at), gs * n, D).transpose(0, 1)
    return o.view(S, Hkv, gs, n, D).permute(0, 3, 1, 2, 4).reshape(S * n, Hq * D).to(s.q.dtype)


def _plain_fork(s, c):
    page, per = c["page"], _ceil(c["rows"], c["page"])
    free, src, dst = c["parents"] * per, [], []
    for i, (kept, shared) in enumerate(_fork_pages(c, s.keeps)):
        p = i // c["children"]
        src.append(p * per * page + np.flatnonzero(s.keeps[p])[shared * page:])
        dst.append(free * page + np.arange(kept - shared * page))
        free += _ceil(kept, page) - shared
    src, dst = (torch.from_numpy(np.concatenate(a)).cuda() for a in (src, dst))
    for p in (s.k_pages, s.v_pages):
        p[:, dst // page, :, dst % page] = p[:, src // page, :, src % page]
    return s.k_pages, s.v_pages


# ------------------------------------------------------------------------ run

def run(s):
    c = s.case
    if own:
        if s.kind == "write":
            return s.step.write(0, s.q, s.k, s.v), s.pool.k, s.pool.v
        if s.kind == "attend":
            return s.step.attend(0, s.q)
        parents = [q for q in s.parents for _ in range(c["children"])]
        keeps = None if c["drop"] == 0 else [k for k in s.keeps for _ in range(c["children"])]
        for q in s.pool.fork(parents, keep=keeps):
            q.free()
        return s.pool.k, s.pool.v
    if s.kind == "write":
        return _plain_write(s, c)
    return _plain_attend(s, c) if s.kind == "attend" else _plain_fork(s, c)


def work(case):
    Hkv, D = case["Hkv"], case["D"]
    if case["kind"] == "write":                                  # rows in, q and the cache rows out
        values = case["S"] * case["n"] * (case["Hq"] + 2 * Hkv) * D
        return {"bytes": values * (SIZE[case["x"]] + SIZE[case["kv"]]), "flops": 3.0 * values}
    if case["kind"] == "attend":
        own_, n = _own_rows(case), case["n"]
        rows = case["system"] + case["groups"] * case["shared"] + sum(own_)
        pairs = sum(n * (case["system"] + case["shared"] + r - n) + n * (n + 1) // 2 for r in own_)
        return {"bytes": 2 * (rows * 2 * Hkv * D + case["S"] * n * 2 * case["Hq"] * D), "flops": 4.0 * D * case["Hq"] * pairs}
    copied = [kept - shared * case["page"] for kept, shared in _fork_pages(case, _keeps(case, 0))]
    read = sum(copied[:: case["children"]])                      # a parent's rows are read once for all its children
    return {"bytes": (read + sum(copied)) * case["L"] * 2 * Hkv * D * 2, "flops": 0}


# ---------------------------------------------------------------------- exact

def exact(case, seed):
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    if case["kind"] == "write":
        q, k, v, pos = _qkv(case, seed)
        axis = _pair_axis(case)
        p = pos[np.zeros(D // 2, int) if axis is None else axis.astype(int)].T.astype(np.float64)   # [M, D/2]
        turn = np.exp(1j * p * THETA ** (-np.arange(0, D, 2) / D))
        turn = torch.from_numpy(turn).cuda()[:, None]

        def rotated(x, heads):
            x = x.double().reshape(-1, heads, 2, D // 2)
            z = torch.complex(x[:, :, 0], x[:, :, 1]) * turn
            return torch.cat([z.real, z.imag], -1)

        S, n, past = case["S"], case["n"], case["past"]
        head, all_ = _ceil(past, page), _ceil(past + n, page)
        pages = [torch.zeros((1, S * (all_ + 1), Hkv, page, D), dtype=torch.float64, device="cuda") for _ in range(2)]
        rows = (rotated(k, Hkv), v.double().reshape(-1, Hkv, D))
        for i in range(S):
            mine = list(range(i * head, (i + 1) * head)) + list(range(S * head + i * (all_ - head), S * head + (i + 1) * (all_ - head)))
            for p, r in zip(pages, rows):
                seq = p[0, mine].transpose(1, 2).reshape(all_ * page, Hkv, D)
                seq[past:past + n] = r[i * n:(i + 1) * n]
                p[0, mine] = seq.view(all_, page, Hkv, D).transpose(1, 2)
        return rotated(q, case["Hq"]).reshape(S * n, -1), pages[0], pages[1]
    if case["kind"] == "fork":
        per, keeps, out = _ceil(case["rows"], page), _keeps(case, seed), []
        n_pages = case["parents"] * (per * (1 + case["children"]) if case["drop"] else per + case["children"])
        parents = _parent_rows(case, seed)
        for j in range(2):
            pages = torch.zeros((case["L"], Hkv, n_pages * page, D), dtype=torch.float64, device="cuda")
            for i, rows in enumerate(parents):
                pages[:, :, i * per * page:i * per * page + case["rows"]] = rows[j].double()
            at = case["parents"] * per * page
            for i, (kept, shared) in enumerate(_fork_pages(case, keeps)):
                p, skip = i // case["children"], shared * page
                mine = parents[p][j][:, :, torch.from_numpy(keeps[p]).cuda().bool()].double()[:, :, skip:]
                pages[:, :, at:at + kept - skip] = mine
                at += _ceil(kept - skip, page) * page
            out.append(pages.view(case["L"], Hkv, n_pages, page, D).transpose(1, 2))
        return tuple(out)
    if work(case)["flops"] > 4e11:
        return None
    (sys_, grp, mine), q = _segments(case, seed)
    n, gs, out = case["n"], case["Hq"] // Hkv, []
    for i, (r, g, (mask, rows)) in enumerate(zip(_own_rows(case), _group(case), _masks(case, seed))):
        T = case["system"] + case["shared"] + r
        see = np.arange(T)[None, :] <= T - n + np.arange(n)[:, None]
        see = see if mask is None else see & (mask[None] != 0)
        see = torch.from_numpy(see if rows is None else see & (rows != 0)).cuda()
        heads = []
        for h in range(Hkv):
            k, v = (torch.cat([sys_[j][h], grp[j][g, h], mine[j][i, h, :r]]).double() for j in range(2))
            for e in range(gs):
                x = q[i * n:(i + 1) * n, (h * gs + e) * D:(h * gs + e + 1) * D].double()
                z = (x @ k.t().contiguous()) / math.sqrt(D)
                heads.append(torch.softmax(torch.where(see, z, -torch.inf), -1) @ v)
        out.append(torch.cat(heads, 1))
    return torch.cat(out)
