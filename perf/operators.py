"""Timed cases of the KV-cache operators: what a serving step calls on the
paged cache of one rank, whose query- and KV-head ranges are of unequal width.

  extend  blocks, slots and positions for a step's new tokens, from the block
          table and the request lengths
  append  rotary positions on q and k, and k and v into their slots
  attend  attention of the new tokens over the cache: one token a sequence
          (serving), a few (drafts), or whole prompts (replay of sessions
          that were evicted)

A case gives lengths as one number and whether they are ragged; the lengths
of each sequence follow from the case, the values from the seed.
"""
import math

import torch

own = False

# a rank's heads: query range [q0, q1), KV range [k0, k1), query heads per KV head
BASE = dict(op="attend", q0=0, q1=8, k0=0, k1=1, group=8, head_dim=128, block_tokens=16, layout="head",
            dtype="bf16", cache="same", n_seq=8, cached=128, fresh=1, ragged=False, pad=0, pool_percent=112,
            rot=128, interleaved=False, scaling="none", softcap=0.0, window=0, slopes=False)


def _case(name=None, **kw):
    c = dict(BASE, **kw)
    if name:
        c["name"] = name
    return c


TINY = dict(q0=0, q1=2, k0=0, k1=1, group=2, head_dim=64, rot=64, dtype="fp16")           # 4 -> 3, rank 0
DENSE5120 = dict(q0=14, q1=27, k0=2, k1=6, group=5, head_dim=128, rot=128)                 # 40 / 8 heads, 4 -> 3, rank 1
DENSE8192 = dict(q0=10, q1=19, k0=1, k1=3, group=8, head_dim=128, rot=128)                 # 64 / 8 heads, 8 -> 7, rank 1
MOE = dict(q0=11, q1=22, k0=1, k1=3, group=8, head_dim=128, rot=128)                       # 32 / 4 heads, 4 -> 3, rank 1


def listed():
    return [
        # the smallest step: eight short sessions get a token each; launches and host calls are all there is
        _case("extend_few", op="extend", **TINY, cached=127, ragged=True, pad=3),
        # a serving step of the 80-layer workload's 128 sessions at 8192 tokens
        _case("extend_serving", op="extend", **DENSE8192, n_seq=128, cached=8190, ragged=True, pool_percent=112),
        # many long sessions, some of them replayed after an eviction: the table is what counts
        _case("extend_replay", op="extend", **DENSE8192, n_seq=512, cached=24001, fresh=301, ragged=True, pad=77),
        # the smallest step's tokens
        _case("append_few", op="append", **TINY, cached=127, ragged=True, pad=3),
        # a prompt of 8192 tokens, long-context scaling by parts
        _case("append_prompt", op="append", **DENSE5120, n_seq=1, cached=70001, fresh=8192, scaling="parts"),
        # an 8-bit token-major cache, interleaved pairs over a part of the head, ragged prompts
        _case("append_e4m3_part", op="append", q0=8, q1=19, k0=1, k1=3, group=8, head_dim=128, rot=64, interleaved=True,
              cache="e4m3", layout="token", n_seq=9, cached=301, fresh=997, ragged=True, pad=5, scaling="linear"),
        # one token each for eight short sessions: latency
        _case("attend_few", **TINY, cached=127, ragged=True),
        # a serving step of the 80-layer workload: 128 sessions at 8192 tokens, head range cutting two groups
        _case("attend_serving", **DENSE8192, n_seq=128, cached=8191),
        # few very long sessions in an 8-bit cache, token-major: the length has to be split
        _case("attend_long_e4m3", **MOE, cache="e4m3", layout="token", n_seq=3, cached=131000, ragged=True),
        # drafts of three tokens with a window, small heads, odd lengths, a capped score
        _case("attend_drafts", q0=3, q1=16, k0=0, k1=4, group=4, head_dim=64, rot=64, dtype="fp16", n_seq=61, cached=3001,
              fresh=3, ragged=True, pad=4, window=1024, softcap=30.0),
        # a prompt of 8192 tokens behind a cached prefix of the same length: the largest product
        _case("attend_prompt", **DENSE8192, n_seq=1, cached=8192, fresh=8192),
        # replay of evicted sessions: ragged prompts from nothing, with a bias by distance
        _case("attend_replay", **DENSE5120, layout="token", n_seq=6, cached=0, fresh=3500, ragged=True, pad=9, slopes=True),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    """One case of the listed ranges: every size over its logarithm, no dearer than the largest listed ones."""
    while True:
        op = rng.choice(["extend", "append", "attend", "attend"])
        group = rng.choice([1, 2, 3, 4, 5, 7, 8])
        k0 = rng.randint(0, 3)
        n_kv = rng.randint(1, 4)
        q0 = group * k0 + rng.randint(0, group - 1)
        q1 = group * (k0 + n_kv - 1) + rng.randint(1, group)
        if q1 <= q0:
            continue
        hd = rng.choice([64, 128, 128, 80, 256])
        rot = rng.choice([hd, hd, hd // 2])
        c = _case(op=op, q0=q0, q1=q1, k0=k0, k1=k0 + n_kv, group=group, head_dim=hd, rot=rot,
                  block_tokens=rng.choice([8, 16, 16, 32, 64]), layout=rng.choice(["head", "token"]),
                  dtype=rng.choice(["bf16", "bf16", "fp16"]), cache=rng.choice(["same", "same", "e4m3"]),
                  ragged=rng.random() < 0.7, pad=rng.choice([0, 0, rng.randint(1, 40)]),
                  interleaved=rng.random() < 0.5, scaling=rng.choice(["none", "linear", "parts"]))
        if op == "extend":
            c.update(n_seq=_log(rng, 1, 512), cached=_log(rng, 1, 30000), fresh=rng.choice([1, 1, _log(rng, 1, 1000)]))
            if sum(work(c).values()) > sum(work(_case(**EXTEND_MOST)).values()):
                continue
        elif op == "append":
            c.update(n_seq=_log(rng, 1, 128), cached=_log(rng, 1, 100000), fresh=rng.choice([1, _log(rng, 1, 8192)]))
            if c["n_seq"] * c["fresh"] > 8192 or c["n_seq"] * (c["cached"] + c["fresh"]) > 300000:
                continue
        else:
            c.update(n_seq=_log(rng, 1, 128), cached=_log(rng, 1, 131000), fresh=rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 8192)]),
                     softcap=rng.choice([0.0, 0.0, 30.0]), window=rng.choice([0, 0, _log(rng, 100, 8192)]),
                     slopes=rng.random() < 0.25)
            ctx, n_q = c["cached"] + c["fresh"], c["q1"] - c["q0"]
            # what the plain form holds: scores, and K and V in 32 bits for each query head
            if c["n_seq"] * n_q * c["fresh"] * ctx > 9 * 8192 * 16384 or c["n_seq"] * ctx * n_q * c["head_dim"] > 128 * 8192 * 9 * 128:
                continue
        return c


EXTEND_MOST = dict(op="extend", n_seq=512, cached=24001, fresh=301, pad=77)


# ---- sizes that follow from a case ------------------------------------------

def _lengths(c):
    """Tokens in the cache before the step and new ones, for each sequence: the first has the case's numbers, the
    others of a ragged case fewer (down to none)."""
    n = c["n_seq"]
    if not c["ragged"]:
        return [c["cached"]] * n, [c["fresh"]] * n
    return [c["cached"] * (64 - (s * 37) % 64) // 64 for s in range(n)], [c["fresh"] * (16 - (s * 23) % 16) // 16 if c["fresh"] > 1 else 1 for s in range(n)]


def _sizes(c):
    cached, fresh = _lengths(c)
    bt = c["block_tokens"]
    held = [-(-a // bt) for a in cached]
    most = max(-(-(a + b) // bt) for a, b in zip(cached, fresh)) + 1  # a spare column
    wanted = sum(-(-(a + b) // bt) for a, b in zip(cached, fresh))
    pool = max(wanted * c["pool_percent"] // 100, wanted)
    return cached, fresh, held, most, pool, sum(fresh) + c["pad"]


def work(c):
    cached, fresh, held, most, pool, rows = _sizes(c)
    hd, n_q = c["head_dim"], c["q1"] - c["q0"]
    n_kv = -(-c["q1"] // c["group"]) - c["q0"] // c["group"]
    ce = 1 if c["cache"] == "e4m3" else 2
    if c["op"] == "extend":  # the table in and out, lengths, starts, a slot and a position for each token
        return {"bytes": 8 * c["n_seq"] * most + 12 * c["n_seq"] + 12 * rows + 20, "flops": 0}
    if c["op"] == "append":
        t, kv = sum(fresh), c["k1"] - c["k0"]
        return {"bytes": t * (hd * (4 * n_q + 2 * (2 + ce) * kv) + 12), "flops": 3 * t * c["rot"] * (n_q + kv)}
    seen = pairs = 0
    for a, f in zip(cached, fresh):
        if not f:
            continue
        w = c["window"] or a + f
        seen += min(a + f, w + f - 1)
        # row i sees min(a + i + 1, w) tokens
        full = max(0, min(f, w - a))  # rows that see everything before them
        pairs += full * a + full * (full + 1) // 2 + (f - full) * w
    return {"bytes": seen * n_kv * hd * 2 * ce + sum(fresh) * n_q * (hd * 4 + 4) + 4 * c["n_seq"] * most, "flops": 4 * hd * n_q * pairs}


# ---- inputs -------------------------------------------------------------------

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


def _rope(c):
    """(base, scaling, factor, low, high, original, amplitude)"""
    if c["scaling"] == "linear":
        return 10000.0, "linear", 4.0, 0.0, 0.0, 0.0, 1.0
    if c["scaling"] == "parts":
        return 1e6, "parts", 8.0, 1.0, 32.0, 8192.0, 0.1 * math.log(8.0) + 1
    return 10000.0, "none", 1.0, 0.0, 0.0, 0.0, 1.0


def _arena(c, g, dev, pool):
    """One layer's arena [K,V][block] and its blocks in the cache's order, with values of a unit spread."""
    n_kv, bt, hd = c["k1"] - c["k0"], c["block_tokens"], c["head_dim"]
    shape = (2, pool, n_kv, bt, hd) if c["layout"] == "head" else (2, pool, bt, n_kv, hd)
    x = torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(generator=g)
    if c["cache"] == "e4m3":
        return (x * 32).to(torch.float8_e4m3fn)
    return x.to(TYPES[c["dtype"]])


def prepare(case, seed):
    c = case
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    cached, fresh, held, most, pool, rows = _sizes(c)
    n, n_q, n_kv, hd, bt = c["n_seq"], c["q1"] - c["q0"], c["k1"] - c["k0"], c["head_dim"], c["block_tokens"]
    s = {"case": c, "rows": rows}
    s["cached"] = torch.tensor(cached, dtype=torch.int32, device=dev)
    s["fresh"] = torch.tensor(fresh, dtype=torch.int32, device=dev)
    # blocks of a pool in use for a while: each session's lie anywhere in it
    ids = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
    have = torch.tensor(held, device=dev)
    if c["op"] != "extend":
        have = torch.tensor([-(-(a + b) // bt) for a, b in zip(cached, fresh)], device=dev)
    at = torch.arange(most, device=dev)[None, :]
    off = (torch.cumsum(have, 0) - have)[:, None] + at
    s["table"] = torch.where(at < have[:, None], ids[off.clamp(max=pool - 1)], -1).to(torch.int32).contiguous()
    s["pool"] = pool
    starts = torch.zeros(n + 1, dtype=torch.int32, device=dev)
    starts[1:] = torch.cumsum(s["fresh"], 0)
    if c["op"] == "extend":
        s["new_table"] = torch.empty_like(s["table"])
        s["starts"] = torch.empty(n + 1, dtype=torch.int32, device=dev)
        s["slots"] = torch.empty(rows, dtype=torch.int64, device=dev)
        s["positions"] = torch.empty(rows, dtype=torch.int32, device=dev)
    else:
        s["new_table"], s["starts"] = s["table"], starts
        t = torch.arange(rows, device=dev, dtype=torch.int32)
        seq = torch.searchsorted(starts[1:], t, right=True).clamp(max=n - 1)
        pos = s["cached"][seq] + t - starts[seq]
        real = t < starts[n]
        slot = s["table"][seq, (pos // bt).clamp(max=most - 1).long()].long() * bt + pos % bt
        s["slots"] = torch.where(real, slot, -1).contiguous()
        s["positions"] = torch.where(real, pos, 0).to(torch.int32).contiguous()
        dt = TYPES[c["dtype"]]
        s["arena"] = _arena(c, g, dev, pool)
        s["scales"] = None
        if c["cache"] == "e4m3":
            s["scales"] = (torch.rand(2, n_kv, generator=g, device=dev) + 0.5) / 32
        if c["op"] == "append":  # one projection's rows: q, k and v side by side
            s["qkv"] = torch.empty(rows, (n_q + 2 * n_kv) * hd, dtype=dt, device=dev).normal_(generator=g)
            s["q_out"] = torch.zeros(rows, n_q, hd, dtype=dt, device=dev)
        else:
            s["q"] = torch.empty(rows, n_q, hd, dtype=dt, device=dev).normal_(generator=g)
            s["out"] = torch.zeros(rows, n_q, hd, dtype=dt, device=dev)
            s["lse"] = torch.zeros(rows, n_q, dtype=torch.float32, device=dev)
            s["slopes"] = None
            if c["slopes"]:
                s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / 64) / 16 for h in range(c["q0"], c["q1"])], device=dev)
    s["status"] = torch.zeros(4, dtype=torch.int32, device=dev)
    if own:  # the handles that a program keeps beside its cache: descriptions and a workspace
        from paper_2511_11617_amd import atp
        arena = s.get("arena")
        arena = torch.empty(256, dtype=torch.uint8, device=dev) if arena is None else arena
        s["cache"] = atp.KVCache(arena=arena.data_ptr() if c["op"] != "extend" else 0,
                                 arena_bytes=arena.numel() * arena.element_size() if c["op"] != "extend" else 0,
                                 num_layers=1, block_tokens=bt, head_dim=hd,
                                 layout=atp.KV_HEAD_MAJOR if c["layout"] == "head" else atp.KV_TOKEN_MAJOR,
                                 num_blocks=pool, q_heads=(c["q0"], c["q1"]), kv_heads=(c["k0"], c["k1"]), group=c["group"],
                                 dtype=atp.BF16 if c["dtype"] == "bf16" else atp.FP16,
                                 cache_dtype=atp.E4M3 if c["cache"] == "e4m3" else None,
                                 scales=s["scales"].data_ptr() if s.get("scales") is not None else 0)
        s["step"] = atp.KVStep(block_table=s["new_table"].data_ptr(), n_seq=n, max_blocks=most, cached=s["cached"].data_ptr(),
                               fresh=s["fresh"].data_ptr(), starts=s["starts"].data_ptr(), slots=s["slots"].data_ptr(),
                               positions=s["positions"].data_ptr(), max_tokens=rows, max_fresh=max(fresh),
                               max_ctx=max(a + b for a, b in zip(cached, fresh)), status=s["status"].data_ptr())
        if c["op"] == "append":
            base, scaling, factor, low, high, original, amplitude = _rope(c)
            s["rope"] = atp.Rope(rot_dim=c["rot"], interleaved=c["interleaved"], base=base,
                                 scaling={"none": atp.ROPE_PLAIN, "linear": atp.ROPE_LINEAR, "parts": atp.ROPE_PARTS}[scaling],
                                 factor=factor, low=low, high=high, original=original, amplitude=amplitude)
        if c["op"] == "attend":
            s["mask"] = atp.Mask(scale=hd ** -0.5, softcap=c["softcap"], window=c["window"],
                                 slopes=s["slopes"].data_ptr() if c["slopes"] else 0)
        need = {"extend": atp.kv_extend_workspace, "attend": atp.kv_attend_workspace}.get(c["op"])
        s["ws_bytes"] = need(s["cache"], s["step"]) if need else 0
        s["ws"] = torch.empty(max(s["ws_bytes"], 256), dtype=torch.uint8, device=dev)
    return s


# ---- one pass -------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"extend": _own_extend, "append": _own_append, "attend": _own_attend}[op](s)
    return {"extend": _plain_extend, "append": _plain_append, "attend": _plain_attend}[op](s)


def _own_extend(s):
    from paper_2511_11617_amd import atp
    atp.kv_extend(s["cache"], s["step"], s["table"].data_ptr(), s["ws"].data_ptr(), s["ws_bytes"],
                  torch.cuda.current_stream().cuda_stream)
    return s["new_table"], s["starts"], s["slots"], s["positions"], s["status"]


def _own_append(s):
    from paper_2511_11617_amd import atp
    c = s["case"]
    hd, n_q, n_kv = c["head_dim"], c["q1"] - c["q0"], c["k1"] - c["k0"]
    p, row = s["qkv"].data_ptr(), (n_q + 2 * n_kv) * hd
    atp.kv_append(s["cache"], s["step"], 0, s["rope"], p, row, p + 2 * n_q * hd, row, p + 2 * (n_q + n_kv) * hd, row,
                  s["q_out"].data_ptr(), n_q * hd, torch.cuda.current_stream().cuda_stream)
    return s["q_out"], s["arena"]


def _own_attend(s):
    from paper_2511_11617_amd import atp
    c = s["case"]
    row = (c["q1"] - c["q0"]) * c["head_dim"]
    atp.kv_attend(s["cache"], s["step"], 0, s["mask"], s["q"].data_ptr(), row, s["out"].data_ptr(), row, s["lse"].data_ptr(),
                  s["ws"].data_ptr(), s["ws_bytes"], torch.cuda.current_stream().cuda_stream)
    return s["out"], s["lse"]


def _plain_extend(s):
    c, dev = s["case"], s["table"].device
    n, bt, pool, table = c["n_seq"], c["block_tokens"], s["pool"], s["table"]
    cached, fresh = s["cached"].long(), s["fresh"].long()
    used = torch.zeros(pool + 1, dtype=torch.bool, device=dev)
    used[torch.where(table < 0, pool, table).reshape(-1).long()] = True
    used[pool] = True
    # the k-th free id, in ascending order
    rank = torch.cumsum(~used, 0) - 1
    free = torch.zeros(pool + 2, dtype=torch.int32, device=dev)
    free[torch.where(used, pool + 1, rank)] = torch.arange(pool + 1, dtype=torch.int32, device=dev)
    b = torch.arange(table.shape[1], device=dev)[None, :]
    want = (b >= (cached // bt)[:, None]) & (b < ((cached + fresh + bt - 1) // bt)[:, None]) & (fresh > 0)[:, None] & (table < 0)
    k = (torch.cumsum(want.reshape(-1), 0) - 1).reshape(want.shape)
    new = torch.where(want, free[k.clamp(min=0)], table)
    starts = torch.zeros(n + 1, dtype=torch.int32, device=dev)
    starts[1:] = torch.cumsum(fresh, 0)
    t = torch.arange(s["rows"], device=dev, dtype=torch.int32)
    seq = torch.searchsorted(starts[1:], t, right=True).clamp(max=n - 1)
    pos = cached[seq] + t - starts[seq]
    real = t < starts[n]
    slot = new[seq, torch.where(real, pos // bt, 0)].long() * bt + pos % bt
    taken = want.sum()
    status = torch.stack([torch.zeros_like(taken), starts[n].long(), taken, (~used).sum() - taken]).to(torch.int32)
    return new, starts, torch.where(real, slot, -1), torch.where(real, pos, 0).to(torch.int32), status


def _plain_append(s):
    c = s["case"]
    hd, rot, n_q, n_kv, bt = c["head_dim"], c["rot"], c["q1"] - c["q0"], c["k1"] - c["k0"], c["block_tokens"]
    base, scaling, factor, low, high, original, amplitude = _rope(c)
    dev, dt = s["qkv"].device, s["qkv"].dtype
    inv = base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=dev) / rot)
    if scaling == "linear":
        inv = inv / factor
    elif scaling == "parts":
        keep = ((original * inv / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        inv = inv * keep + inv / factor * (1 - keep)
    angle = s["positions"].double()[:, None] * inv  # a far position's angle needs more than 32 bits
    cos, sin = ((f(angle) * amplitude).float()[:, None, :] for f in (torch.cos, torch.sin))
    rows = s["qkv"].float().reshape(s["rows"], n_q + 2 * n_kv, hd)
    qk, v = rows[:, :n_q + n_kv], rows[:, n_q + n_kv:]
    if c["interleaved"]:
        x, y = qk[..., 0:rot:2], qk[..., 1:rot:2]
        turned = torch.stack([x * cos - y * sin, y * cos + x * sin], -1).flatten(-2)
    else:
        x, y = qk[..., :rot // 2], qk[..., rot // 2:rot]
        turned = torch.cat([x * cos - y * sin, y * cos + x * sin], -1)
    qk = torch.cat([turned, qk[..., rot:]], -1)
    real = s["slots"] >= 0
    q = torch.where(real[:, None, None], qk[:, :n_q].to(dt), s["q_out"])
    kv = torch.stack([qk[:, n_q:], v])  # [2, rows, heads, hd]
    if s["scales"] is not None:
        kv = (kv / s["scales"][:, None, :, None]).clamp(-448, 448)
    n_real = s["rows"] - c["pad"]  # the padding is behind the real tokens
    kv = kv[:, :n_real].to(s["arena"].dtype)
    block, off = s["slots"][:n_real] // bt, s["slots"][:n_real] % bt
    bits = s["arena"].view(torch.uint8) if s["scales"] is not None else s["arena"]
    kv = kv.view(torch.uint8) if s["scales"] is not None else kv
    if c["layout"] == "head":
        bits[:, block, :, off] = kv.transpose(0, 1)
    else:
        bits[:, block, off] = kv
    return q, s["arena"]


def _plain_attend(s):
    c = s["case"]
    hd, n_q, bt, n = c["head_dim"], c["q1"] - c["q0"], c["block_tokens"], c["n_seq"]
    dev, dt = s["q"].device, s["q"].dtype
    cached, fresh = _lengths(c)
    ctx, most = max(a + b for a, b in zip(cached, fresh)), max(fresh)
    t = torch.arange(ctx, device=dev)
    block = s["table"][:, t // bt].long()  # [n, ctx]
    there = (block >= 0) & (t[None, :] < (s["cached"] + s["fresh"])[:, None])
    head = torch.arange(c["q0"], c["q1"], device=dev) // c["group"] - c["k0"]
    block = block.clamp(min=0)

    def rows_of(which):  # [n, n_q, ctx, hd] in 32 bits
        a = s["arena"][which]
        if s["scales"] is not None:
            a = a.view(torch.uint8)
        a = a[block, :, t % bt] if c["layout"] == "head" else a[block, t % bt]  # [n, ctx, n_kv, hd]
        if s["scales"] is not None:
            a = a.view(torch.float8_e4m3fn).float() * s["scales"][which][:, None]
        return a.float()[:, :, head].transpose(1, 2).contiguous()

    i = torch.arange(most, device=dev)
    real = i[None, :] < s["fresh"][:, None]  # [n, most]
    row = (s["starts"][:-1, None] + i[None, :]).clamp(max=s["rows"] - 1).long()
    q = s["q"][row].float().transpose(1, 2).contiguous()  # [n, n_q, most, hd]
    score = torch.matmul(q, rows_of(0).transpose(2, 3).contiguous()).mul_(hd ** -0.5)
    if c["softcap"]:
        score = score.div_(c["softcap"]).tanh_().mul_(c["softcap"])
    away = (s["cached"][:, None] + i[None, :])[:, :, None] - t[None, None, :]  # [n, most, ctx]
    if s["slopes"] is not None:
        score -= s["slopes"][:, None, None] * away[:, None].float()
    seen = (away >= 0) & there[:, None, :] & real[:, :, None]
    if c["window"]:
        seen &= away < c["window"]
    score.masked_fill_(~seen[:, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight, rows_of(1)) / total.clamp(min=1e-38)
    lse = (top + total.log()).squeeze(-1)
    got, got_lse = s["out"].clone(), s["lse"].clone()
    got[row[real]] = out.transpose(1, 2)[real].to(dt)
    got_lse[row[real]] = lse.transpose(1, 2)[real]
    return got, got_lse


# ---- the definitions in 64 bits -----------------------------------------------

def exact(case, seed):
    if case["op"] == "extend":
        return None  # whole numbers only
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attend(s)


def _exact_append(s):
    """Each pair as a complex number, turned by exp(i angle)."""
    c = s["case"]
    hd, rot, bt = c["head_dim"], c["rot"], c["block_tokens"]
    n_q, n_kv = c["q1"] - c["q0"], c["k1"] - c["k0"]
    base, scaling, factor, low, high, original, amplitude = _rope(c)
    turns = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            r = original * f / (2 * math.pi)
            keep = 0.0 if r < low else 1.0 if r > high else (r - low) / (high - low)
            f = (1 - keep) * f / factor + keep * f
        turns.append(f)
    real = [i for i in range(s["rows"]) if i < s["rows"] - c["pad"]]
    x = s["qkv"].double().reshape(s["rows"], n_q + 2 * n_kv, hd)
    pos = s["positions"].double()
    turn = torch.polar(torch.full_like(pos, amplitude)[:, None].expand(-1, rot // 2).contiguous(),
                       pos[:, None] * torch.tensor(turns, dtype=torch.float64, device=pos.device))
    for h in range(n_q + n_kv):
        part = x[:, h, :rot]
        re, im = (part[:, 0::2], part[:, 1::2]) if c["interleaved"] else (part[:, :rot // 2], part[:, rot // 2:])
        z = torch.complex(re.contiguous(), im.contiguous()) * turn
        if c["interleaved"]:
            x[:, h, 0:rot:2], x[:, h, 1:rot:2] = z.real, z.imag
        else:
            x[:, h, :rot] = torch.cat([z.real, z.imag], 1)
    q = s["q_out"].double()
    q[:len(real)] = x[:len(real), :n_q]
    arena = s["arena"].double()
    block, off = s["slots"][:len(real)] // bt, s["slots"][:len(real)] % bt
    for which in range(2):
        for h in range(n_kv):
            val = x[:len(real), n_q + which * n_kv + h]
            if s["scales"] is not None:
                val = (val / s["scales"][which, h].double()).clamp(-448, 448)
            if c["layout"] == "head":
                arena[which, :, h][block, off] = val
            else:
                arena[which, :, :, h][block, off] = val
    return q, arena


def _exact_attend(s):
    """Sequence by sequence and head by head, over the visible tokens."""
    c = s["case"]
    hd, bt = c["head_dim"], c["block_tokens"]
    cached, fresh = _lengths(c)
    out, lse = s["out"].double(), s["lse"].double()
    row = 0
    dev = out.device
    for q_seq, (a, f) in enumerate(zip(cached, fresh)):
        if not f:
            continue
        t = torch.arange(a + f, device=dev)
        block = s["table"][q_seq, t // bt].long()
        for h in range(c["q0"], c["q1"]):
            kh = h // c["group"] - c["k0"]
            K, V = ((s["arena"][w][:, kh] if c["layout"] == "head" else s["arena"][w][:, :, kh]) for w in range(2))
            if s["scales"] is not None:
                K, V = K.view(torch.uint8), V.view(torch.uint8)
            K, V = K[block, t % bt], V[block, t % bt]
            if s["scales"] is not None:
                K, V = (x.view(torch.float8_e4m3fn).double() * s["scales"][w, kh].double() for w, x in enumerate((K, V)))
            K, V = K.double(), V.double()
            for lo in range(0, f, 2048):  # rows, some at a time
                hi = min(f, lo + 2048)
                away = torch.arange(a + lo, a + hi, device=dev)[:, None] - t[None, :]
                z = s["q"][row + lo:row + hi, h - c["q0"]].double() @ K.T.contiguous() / math.sqrt(hd)
                if c["softcap"]:
                    z = c["softcap"] * torch.tanh(z / c["softcap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][h - c["q0"]].double() * away
                z = torch.where((away >= 0) & (away < (c["window"] or a + f)), z, -math.inf)
                l = torch.logsumexp(z, 1)
                lse[row + lo:row + hi, h - c["q0"]] = l
                out[row + lo:row + hi, h - c["q0"]] = torch.exp(z - l[:, None]) @ V
        row += f
    return out, lse
