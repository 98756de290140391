"""Performance cases of the key-value cache operators, through the public Python API.

A case is one step that a serving program makes with ``api.KvCache``, a paged
cache of keys and values held in 8 bits with one scale for each block of tokens
and head:

- ``append``: new rows of many sequences quantised into their blocks (a decode
  step's single tokens, draft tokens written again over rejected ones, whole
  prompts), and the rows of the blocks that changed read back;
- ``decode``: attention of one or a few query tokens of each sequence over what
  it holds, with the weight that each block received added up where eviction
  will ask for it;
- ``chunk``: attention of a chunk of a prompt over the cache it was appended to;
- ``evict``: a cache at its budget takes new blocks and gives up as many, those
  that have received the least attention weight.

Rows are N(0, 1) in bf16, as in the MoE layer's cases; 16 query heads of 128
make the layer's 2,048 columns.  Lengths are ragged, blocks lie in any order.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# dim, query heads, key-value heads: 2,048 or 4,096 query columns, and a narrow layer's 256
WIDE = {"heads": 16, "kv_heads": 2, "dim": 128}
TALL = {"heads": 16, "kv_heads": 2, "dim": 256}
NARROW = {"heads": 4, "kv_heads": 4, "dim": 64}


def _case(kind, name=None, *, seqs, length, new, shape=WIDE, block=32, fmt="q8", softcap=0.0, window=0, observe=False,
          keep=0):
    c = {"kind": kind, "seqs": seqs, "length": length, "new": new, **shape, "block": block, "format": fmt,
         "softcap": softcap, "window": window, "observe": observe, "keep": keep}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a decode step of a full batch: one row a sequence, its block quantised again
        _case("append", "append_64x1", seqs=64, length=8192, new=1),
        # a batch of prompts of any length enters, in the floating format
        _case("append", "append_5x3000_e4m3", seqs=5, length=3000, new=3000, shape=TALL, block=64, fmt="e4m3"),
        # the longest prompt of the layer's cases at once
        _case("append", "append_1x32768", seqs=1, length=32768, new=32768),
        # one conversation, short: launches and latency
        _case("decode", "decode_1x1000", seqs=1, length=1000, new=1),
        # one conversation at the longest prompt's end
        _case("decode", "decode_1x32768", seqs=1, length=32768, new=1),
        # a full batch of conversations whose caches are near their budget: block weights are kept
        _case("decode", "decode_64x8192_observe", seqs=64, length=8192, new=1, observe=True),
        # tall heads, capped scores, floating format, four draft tokens to verify
        _case("decode", "decode_12x20000_draft4", seqs=12, length=20000, new=4,
              shape={"heads": 8, "kv_heads": 2, "dim": 256}, block=64, fmt="e4m3", softcap=50.0),
        # a narrow layer's batch of short prompts, one head a group, windowed
        _case("chunk", "chunk_8x500_narrow", seqs=8, length=500, new=500, shape=NARROW, block=16, window=200),
        # prompts of any length from their first token
        _case("chunk", "chunk_4x3000_e4m3", seqs=4, length=3000, new=3000, shape=TALL, block=64, fmt="e4m3",
              softcap=50.0),
        # the last chunk of the longest prompt
        _case("chunk", "chunk_4096_of_32768", seqs=1, length=32768, new=4096),
        # caches at their budget take a block and give one up
        _case("evict", "evict_64x256", seqs=64, length=8192, new=32, keep=256),
        _case("evict", "evict_3x4000", seqs=3, length=64000, new=64, block=16, keep=4000),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Any batch, length, head layout, block and format of the same kinds;
    totals stay below those of the largest listed cases."""
    kind = rng.choice(["append", "decode", "decode", "chunk", "chunk", "evict"])
    kv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 3, 4, 6, 7, 8])
    dim = rng.choice([64, 128, 256])
    shape = {"heads": kv * group, "kv_heads": kv, "dim": dim}
    kw = {"shape": shape, "block": rng.choice([16, 32, 64, 128]), "fmt": rng.choice(["q8", "e4m3"])}
    budget = 64 * 8192 * 2 * 128 // (kv * dim)  # cached tokens in all
    if kind == "append":
        seqs = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, max(1, min(32768, 32768 * 256 // (seqs * kv * dim))))
        return _case(kind, seqs=seqs, length=new + rng.choice([0, rng.randint(1, 4000)]), new=new, **kw)
    if kind == "evict":
        seqs = _log_int(rng, 1, 64)
        keep = _log_int(rng, 8, max(8, min(4000, budget // (seqs * kw["block"]))))
        return _case(kind, seqs=seqs, length=keep * kw["block"], new=kw["block"] * rng.randint(1, 3), keep=keep, **kw)
    score = {"softcap": rng.choice([0.0, 0.0, 30.0]), "window": rng.choice([0, 0, 0, 777])}
    if kind == "decode":
        seqs = _log_int(rng, 1, 64)
        length = _log_int(rng, 1, max(1, min(32768, budget // seqs)))
        new = min(length, rng.choice([1, 1, 1, 2, 3]))
        return _case(kind, seqs=seqs, length=length, new=new, observe=rng.random() < 0.5, **score, **kw)
    seqs = _log_int(rng, 1, 8)
    length = _log_int(rng, 33, max(33, min(32768, budget // (4 * seqs))))
    most = min(length, 4096 * 32768 * 16 * 128 // (2 * seqs * length * kv * group * dim))
    return _case(kind, seqs=seqs, length=length, new=max(1, min(most, _log_int(rng, 33, 4096))), **score, **kw)


# --------------------------------------------------------------------------
# the case's lengths (plain numbers, the same for every seed)
# --------------------------------------------------------------------------
def _lens(case):
    """(tokens held by each sequence after the step's rows, new rows of each)."""
    B, L, n, P = case["seqs"], case["length"], case["new"], case["block"]
    if case["kind"] == "evict":
        return np.full(B, case["keep"] * P, np.int64), np.full(B, n, np.int64)
    r = np.random.RandomState((B * 1000003 + L * 101 + n) % (1 << 31))
    new = np.where(n >= 33, r.randint(max(1, n // 3), n + 1, B), n)
    new[0] = n
    if L == n:
        return new.copy(), new
    held = r.randint(max(1, L // 4), L + 1, B)
    held[0] = L
    return np.maximum(held, new), new


def _gen(*key):
    return torch.Generator(device="cuda").manual_seed(int(np.random.SeedSequence(key).generate_state(1, np.uint64)[0] >> 1))


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _quantise(x, fmt):
    """[..., P, D] rows of blocks -> (codes uint8, scale fp32 [...]), in 32 bits:
    scale = amax / top, code = x * (top / amax) rounded; 8-bit codes are offset by 128."""
    top = 127.0 if fmt == "q8" else 448.0
    amax = x.abs().amax((-1, -2)).clamp_min(1e-20)
    scale = amax * float(np.float32(1) / np.float32(top))
    y = x * (torch.full_like(amax, top) / amax)[..., None, None]
    if fmt == "q8":
        return (torch.round(y).clamp(-127, 127) + 128).to(torch.uint8), scale
    return y.to(torch.float8_e4m3fn).view(torch.uint8), scale


def _values(codes, fmt):
    return codes.float() - 128 if fmt == "q8" else codes.view(torch.float8_e4m3fn).float()


def _held_rows(case, seed, at):
    """bf16 [2, B, L, kv_heads, dim]: keys and values of the tokens held before
    (append, evict) or at (decode, chunk) the call; the longest sequence's L."""
    return torch.randn((2, case["seqs"], max(at, 1), case["kv_heads"], case["dim"]), generator=_gen(seed, 1),
                       device="cuda", dtype=torch.bfloat16)


def _new_rows(case, seed, n):
    """The step's rows: keys and values, or queries in the first's place."""
    gen, D = _gen(seed, 2), case["dim"]
    if case["kind"] in ("decode", "chunk"):
        return torch.randn((n, case["heads"], D), generator=gen, device="cuda", dtype=torch.bfloat16), None
    kv = torch.randn((n, 2, case["kv_heads"], D), generator=gen, device="cuda", dtype=torch.bfloat16)
    return kv[:, 0], kv[:, 1]  # slices of one projection's output: rows with a stride


def _block_weights(case, seed, n):
    return torch.rand((n,), generator=_gen(seed, 3), device="cuda") * 4


def _order(seed, n):
    return np.random.default_rng([seed, 4]).permutation(n)


def prepare(case, seed):
    """A cache in use: each sequence's blocks filled, its table, its latest rows
    in 16 bits, the pool's free blocks, and the step's rows."""
    B, P, D, K, fmt = (case[k] for k in ("seqs", "block", "dim", "kv_heads", "format"))
    total, new = _lens(case)
    kind = case["kind"]
    before = total if kind in ("decode", "chunk", "evict") else total - new
    per = int(max(total.max(), 1) + P - 1) // P + (-(-case["new"] // P) + 1 if kind == "evict" else 1)
    n_seqs = B + 2  # more sequences than the step's batch
    n_blocks = int(sum(-(-(t + (case["new"] if kind == "evict" else 0)) // P) for t in total)) + 8
    seqs = np.random.default_rng([seed, 5]).permutation(n_seqs)[:B]
    order = _order(seed, n_blocks)
    rows = _held_rows(case, seed, int(before.max()))
    L = rows.shape[2]
    nb = -(-L // P)
    table = np.zeros((n_seqs, per), np.int32)
    state = np.zeros((n_seqs, 4), np.int32)
    at = 0
    src_b, src_j, ids = [], [], []
    for b, s in enumerate(seqs):
        n = int(-(-before[b] // P))
        table[s, :n] = order[at:at + n]
        state[s, 0] = state[s, 1] = before[b]
        state[s, 2] = max(0, (int(before[b]) - 1) // P - 1) * P if before[b] else 0
        src_b.append(np.full(n, b))
        src_j.append(np.arange(n))
        ids.append(order[at:at + n])
        at += n
    # the pool, and one block past it where the plain form puts what it does not keep
    codes = torch.full((2, n_blocks + 1, K, P, D), 128 if fmt == "q8" else 0, dtype=torch.uint8, device="cuda")
    scale = torch.ones((2, n_blocks + 1, K), device="cuda")
    recent = torch.zeros((n_seqs, 2, K, 2 * P, D), dtype=torch.bfloat16, device="cuda")
    if at:
        live = torch.arange(L, device="cuda")[None] < torch.tensor(before, device="cuda")[:, None]
        for w in range(2):
            x = torch.zeros((B, nb * P, K, D), device="cuda")
            x[:, :L] = rows[w].float() * live[..., None, None]
            x = x.view(B, nb, P, K, D).transpose(2, 3)
            c, s = _quantise(x, fmt)
            where = torch.tensor(np.concatenate(ids).astype(np.int64), device="cuda")
            fb, fj = (torch.tensor(np.concatenate(v), device="cuda") for v in (src_b, src_j))
            codes[w, where], scale[w, where] = c[fb, fj], s[fb, fj]
            del x, c, s
        for b, s in enumerate(seqs):
            lo = int(state[s, 2])
            pos = torch.arange(lo, int(before[b]), device="cuda")
            recent[int(s)][:, :, pos % (2 * P)] = rows[:, b, lo:int(before[b])].transpose(1, 2)
    free = np.zeros(n_blocks, np.int32)
    free[:n_blocks - at] = order[at:][::-1]
    N = int(new.sum())
    x, y = _new_rows(case, seed, N)
    st = {"case": case, "seqs": _ints(seqs), "cu": _ints(np.concatenate([[0], np.cumsum(new)])), "rows": N,
          "max_new": int(new.max()), "x": x, "y": y, "start": _ints(before),
          "codes": codes, "scale": scale, "recent": recent, "table": _ints(table), "seq_state": _ints(state),
          "free_ids": _ints(free), "control": _ints([n_blocks - at] + [0] * 7),
          "weight": _block_weights(case, seed, n_blocks + 1), "blocks": nb}
    if kind == "evict":
        st["first"], st["max_read"] = None, int(new.max())
    else:  # what an append reads back: the blocks that it changed
        first = before // P * P
        st["first"], st["max_read"] = _ints(first), int((total - first).max())
        st["cu_read"], st["rows_read"] = _ints(np.concatenate([[0], np.cumsum(total - first)])), int((total - first).sum())
    if own:
        from paper_2608_23805_gb300 import api
        from paper_2608_23805_gb300 import native as N_
        st["cache"] = api.KvCache(n_seqs=n_seqs, max_blocks=per, n_blocks=n_blocks, n_kv_heads=K, head_dim=D,
                                  block_tokens=P, fmt=N_.MSI_KV_Q8 if fmt == "q8" else N_.MSI_KV_E4M3,
                                  buffers={"k_codes": codes[0, :n_blocks], "v_codes": codes[1, :n_blocks],
                                           "k_scale": scale[0, :n_blocks], "v_scale": scale[1, :n_blocks],
                                           "recent": recent, "table": st["table"], "seq_state": st["seq_state"],
                                           "free_ids": st["free_ids"], "control": st["control"],
                                           "weight": st["weight"][:n_blocks]})
    return st


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    case, cache = s["case"], s["cache"]
    if case["kind"] == "append":
        cache.append(s["x"], s["y"], s["cu"], seqs=s["seqs"], start=s["start"])
        k, v = cache.read(s["cu_read"], s["rows_read"], seqs=s["seqs"], first=s["first"])
        return {"k": k, "v": v, "state": s["seq_state"]}
    if case["kind"] == "evict":
        cache.append(s["x"], s["y"], s["cu"], seqs=s["seqs"])
        cache.evict(s["seqs"], keep=case["keep"], sinks=1, recent=2)
        return {"table": s["table"], "state": s["seq_state"], "free": s["free_ids"], "control": s["control"][:2],
                "weight": s["weight"][:-1]}
    out, lse = cache.attention(s["x"], s["cu"], s["max_new"], seqs=s["seqs"], softcap=case["softcap"],
                               window=case["window"], observe=case["observe"])
    return {"out": out, "lse": lse, **({"weight": s["weight"][:-1]} if case["observe"] else {})}


# --------------------------------------------------------------------------
# the plain form: elementary torch operations in 32 bits
# --------------------------------------------------------------------------
def _run_plain(s):
    case = s["case"]
    if case["kind"] == "append":
        _plain_append(s, s["start"])
        k, v = _plain_read(s)
        return {"k": k, "v": v, "state": s["seq_state"]}
    if case["kind"] == "evict":
        _plain_append(s, s["seq_state"][s["seqs"].long(), 0])
        _plain_evict(s)
        return {"table": s["table"], "state": s["seq_state"], "free": s["free_ids"], "control": s["control"][:2],
                "weight": s["weight"][:-1]}
    return _plain_attention(s)


def _plain_append(s, start):
    """Rows cu[b] .. cu[b+1] become tokens start[b].. of sequence seqs[b]; every
    block that they touch is quantised from its 16-bit rows."""
    case, P = s["case"], s["case"]["block"]
    seqs, cu = s["seqs"].long(), s["cu"].long()
    start = start.long()
    old, pos0 = s["seq_state"][seqs, 0].long(), s["seq_state"][seqs, 1].long()
    new = cu[1:] - cu[:-1]
    end = start + new
    # blocks from the free list's end, in the batch's order
    had, have = (old + P - 1) // P, (end + P - 1) // P
    add = (have - had).clamp_min(0)
    pre = torch.cumsum(add, 0) - add
    m = (s["max_new"] + P - 2) // P + 1
    j = start[:, None] // P + torch.arange(m, device="cuda")  # [B, m] the touched blocks
    touched = j < have[:, None]
    n_free = s["control"][0].long()
    pick = (n_free - 1 - pre[:, None] - (j - had[:, None])).clamp(0, s["free_ids"].numel() - 1)
    col = j.clamp_max(s["table"].shape[1] - 1)
    held = s["table"][seqs[:, None], col].long()
    fresh = touched & (j >= had[:, None])
    ids = torch.where(fresh, s["free_ids"].long()[pick], held)
    s["table"][seqs[:, None], col] = torch.where(touched, ids, held).int()
    spare = s["codes"].shape[1] - 1
    ids = torch.where(touched, ids, spare)
    # each block's rows: new ones, and those that it held
    tok = j[..., None] * P + torch.arange(P, device="cuda")  # [B, m, P]
    is_new = (tok >= start[:, None, None]) & (tok < end[:, None, None])
    is_old = tok < start[:, None, None]
    row = (cu[:-1, None, None] + tok - start[:, None, None]).clamp(0, s["rows"] - 1)
    shift = (pos0 - old)[:, None, None]
    for w, x in enumerate((s["x"], s["y"])):
        ring = s["recent"][seqs[:, None, None], w, :, (tok + shift) % (2 * P)].float()
        rows = torch.where(is_new[..., None, None], x[row].float(), torch.where(is_old[..., None, None], ring, 0.0))
        codes, scale = _quantise(rows.transpose(2, 3), case["format"])
        s["codes"][w, ids] = codes
        s["scale"][w, ids] = scale
        # the last two blocks' rows stay in 16 bits
        r = torch.arange(2 * P, device="cuda")
        last = ((end - 1).clamp_min(0) // P - 1)[:, None] * P + r  # [B, 2P]
        at = (last + (pos0 - old)[:, None]) % (2 * P)
        keep = (last >= start[:, None]) & (last < end[:, None])
        src = (cu[:-1, None] + last - start[:, None]).clamp(0, s["rows"] - 1)
        was = s["recent"][seqs[:, None], w, :, at]
        s["recent"][seqs[:, None], w, :, at] = torch.where(keep[..., None, None], x[src], was)
    s["weight"][torch.where(fresh, ids, spare)] = 0.0
    pos = pos0 - old + end
    start_pos = pos0 - old + start
    kept_from = torch.minimum(s["seq_state"][seqs, 2].long(), start_pos)
    floor = torch.div(pos - 1, P, rounding_mode="floor") * P - P
    s["seq_state"][seqs] = torch.stack([end, pos, torch.maximum(kept_from, floor), torch.zeros_like(end)], 1).int()
    s["control"][0] -= add.sum().int()


def _plain_read(s):
    """Tokens first[b] .. length of each sequence, as bf16 rows."""
    case, P = s["case"], s["case"]["block"]
    seqs, cu = s["seqs"].long(), s["cu_read"].long()
    b = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), cu[1:] - cu[:-1], output_size=s["rows_read"])
    tok = torch.arange(s["rows_read"], device="cuda") - cu[b] + s["first"].long()[b]
    ids = s["table"][seqs[b], tok // P].long()
    return tuple((_values(s["codes"][w, ids, :, tok % P], case["format"]) * s["scale"][w, ids][..., None])
                 .to(torch.bfloat16) for w in range(2))


def _plain_evict(s):
    """Each sequence keeps its first block, its last two, and of the others
    those with the greatest weight (ties: the earlier)."""
    case, P = s["case"], s["case"]["block"]
    keep, n = case["keep"], case["keep"] + case["new"] // case["block"]
    seqs = s["seqs"].long()
    ids = s["table"][seqs, :n].long()
    w = s["weight"][ids]
    at = torch.arange(n, device="cuda")
    w = torch.where((at < 1) | (at >= n - 2), math.inf, w)
    rank = torch.argsort(torch.argsort(w, dim=1, descending=True, stable=True), dim=1)
    kept = rank < keep
    first = torch.argsort((~kept).int(), dim=1, stable=True)  # the kept ones in order, then the others in order
    ids = torch.gather(ids, 1, first)
    s["table"][seqs, :keep] = ids[:, :keep].int()
    gone = ids[:, keep:].reshape(-1).int()
    slot = s["control"][0].long() + torch.arange(gone.numel(), device="cuda")
    s["free_ids"][slot] = gone
    s["control"][0] += gone.numel()
    s["seq_state"][seqs, 0] -= (n - keep) * P


def _plain_attention(s):
    case = s["case"]
    B, P, D, K, fmt = (case[k] for k in ("seqs", "block", "dim", "kv_heads", "format"))
    G, T, n = case["heads"] // K, s["max_new"], s["blocks"]
    seqs, cu = s["seqs"].long(), s["cu"].long()
    length, new = s["seq_state"][seqs, 0].long(), cu[1:] - cu[:-1]
    ids = s["table"][seqs, :n].long()
    live = torch.arange(n, device="cuda") * P < length[:, None]
    ids = torch.where(live, ids, s["codes"].shape[1] - 1)

    def held(w):  # [B, K, n P, D]
        x = _values(s["codes"][w][ids], fmt) * s["scale"][w][ids][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(B, K, n * P, D)

    i = torch.arange(T, device="cuda")
    row = (cu[:-1, None] + i).clamp_max(s["rows"] - 1)
    q = s["x"][row].float().view(B, T, K, G, D).transpose(1, 2).reshape(B, K, T * G, D)
    score = (q @ held(0).transpose(2, 3)).view(B, K, T, G, n * P).mul_(1 / math.sqrt(D))
    if case["softcap"]:
        score.div_(case["softcap"]).tanh_().mul_(case["softcap"])
    last = (length - new)[:, None] + i  # the token that each query row stands at
    tok = torch.arange(n * P, device="cuda")
    seen = (tok <= last[..., None]) & (tok < length[:, None, None])
    if case["window"]:
        seen &= tok > last[..., None] - case["window"]
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp_min(-1e30)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.view(B, K, T * G, n * P) @ held(1)).view(B, K, T, G, D) / total.clamp_min(1e-37)
    lse = (top + torch.log(total))[..., 0]
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), new, output_size=s["rows"])
    i = torch.arange(s["rows"], device="cuda") - cu[b]
    got = {"out": out.permute(0, 2, 1, 3, 4).reshape(B, T, K * G, D)[b, i].to(torch.bfloat16),
           "lse": lse.permute(0, 2, 1, 3).reshape(B, T, K * G)[b, i]}
    if case["observe"]:
        p = p / total.clamp_min(1e-37) * (torch.arange(T, device="cuda") < new[:, None])[:, None, :, None, None]
        w = p.sum((1, 2, 3)).view(B, n, P).sum(2)
        s["weight"].index_add_(0, ids.reshape(-1), torch.where(live, w, 0.0).reshape(-1))
        got["weight"] = s["weight"][:-1]
    return got


# --------------------------------------------------------------------------
def work(case):
    """Cached codes and scales that some query sees read once, rows in and out
    once; 4 flops for each query head, seen token and column."""
    B, P, D, K, H = (case[k] for k in ("seqs", "block", "dim", "kv_heads", "heads"))
    total, new = _lens(case)
    N = float(new.sum())
    token = 2.0 * K * (D + 4.0 / P)  # bytes of one held token
    if case["kind"] == "append":
        first = (total - new) // P * P
        old = float((total - new - first).sum())
        touched = float((total - first).sum())
        # rows in, the touched blocks' codes out; then those codes in and their rows out
        return {"bytes": 4.0 * K * D * (N + old) + 2 * touched * token + touched * 4 * K * D, "flops": 4.0 * touched * K * D}
    if case["kind"] == "evict":
        n = case["keep"] + case["new"] // P
        return {"bytes": N * (4.0 * K * D + token) + B * n * 12.0, "flops": 4.0 * N * K * D}
    pairs, seen = 0.0, 0.0
    for t, n in zip(total.tolist(), new.tolist()):
        last = np.arange(t - n, t, dtype=np.float64)
        see = last + 1 if not case["window"] else np.minimum(last + 1, case["window"])
        pairs += see.sum()
        seen += t - max(0, t - n - case["window"] + 1) if case["window"] else t
    extra = seen / P * 12 if case["observe"] else 0.0
    return {"bytes": float(seen * token + N * H * (4 * D + 4) + extra), "flops": float(4 * pairs * H * D)}


# --------------------------------------------------------------------------
# the same in 64 bits, sequence by sequence
# --------------------------------------------------------------------------
def _exact_block(x, fmt):
    """Values that a block's rows [n, K, D] stand for after rounding, [n, K, D]."""
    top = 127.0 if fmt == "q8" else 448.0
    amax = x.abs().amax((0, 2), keepdim=True).clamp_min(1e-20)
    y = x * (top / amax)
    if fmt == "q8":
        y = torch.round(y)
    else:  # e4m3: 3 bits after the leading one, a spacing of 2^-9 at least
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
        y = (torch.round(y / step) * step).clamp(-448, 448)
    return y * (amax / top)


def _exact_append(case, seed):
    P = case["block"]
    total, new = _lens(case)
    before = total - new
    rows = _held_rows(case, seed, int(before.max()))
    x, y = _new_rows(case, seed, int(new.sum()))
    cu = np.concatenate([[0], np.cumsum(new)])
    got = [[], []]
    for b in range(case["seqs"]):
        first = int(before[b]) // P * P
        for w, fresh in enumerate((x, y)):
            all_ = torch.cat([rows[w, b, first:int(before[b])], fresh[cu[b]:cu[b + 1]]]).double()
            full = all_.shape[0] // P * P
            if full:
                blocks = all_[:full].view(full // P, P, *all_.shape[1:]).transpose(0, 1).reshape(P, -1, all_.shape[2])
                v = _exact_block(blocks, case["format"]).view(P, full // P, *all_.shape[1:]).transpose(0, 1)
                got[w].append(v.reshape(full, *all_.shape[1:]))
            if full < all_.shape[0]:
                got[w].append(_exact_block(all_[full:], case["format"]))
    return {"k": torch.cat(got[0]), "v": torch.cat(got[1]), "state": None}


def exact(case, seed):
    if case["kind"] == "append":
        return _exact_append(case, seed)
    if case["kind"] == "evict":
        return None  # whole numbers, and weights that are moved but not computed
    B, P, D, K, fmt = (case[k] for k in ("seqs", "block", "dim", "kv_heads", "format"))
    G = case["heads"] // K
    total, new = _lens(case)
    rows = _held_rows(case, seed, int(total.max()))
    q, _ = _new_rows(case, seed, int(new.sum()))
    n_blocks = int(sum(-(-t // P) for t in total)) + 8
    weight = _block_weights(case, seed, n_blocks + 1)[:-1].double()
    order = torch.tensor(_order(seed, n_blocks), device="cuda")
    cu = np.concatenate([[0], np.cumsum(new)])
    outs, lses, at = [], [], 0
    for b in range(B):
        L, n = int(total[b]), int(new[b])
        nb = -(-L // P)
        kv = []
        for w in range(2):
            x = torch.zeros((nb * P, K, D), device="cuda")
            x[:L] = rows[w, b, :L].float()
            # the cache's own rounding is an input here: in 32 bits, as prepare() makes it
            c, s = _quantise(x.view(nb, P, K, D).transpose(1, 2), fmt)
            v = (_values(c, fmt).double() * s.double()[..., None, None]).transpose(1, 2)
            kv.append(v.reshape(nb * P, K, D)[:L])
        out = torch.empty((n, K, G, D), dtype=torch.float64, device="cuda")
        lse = torch.empty((n, K, G), dtype=torch.float64, device="cuda")
        per = torch.zeros(nb * P, dtype=torch.float64, device="cuda")
        qs = q[cu[b]:cu[b + 1]].double().view(n, K, G, D)
        tok = torch.arange(L, device="cuda")
        step = max(1, (1 << 28) // (G * L))
        for lo in range(0, n, step):
            hi = min(n, lo + step)
            stand = torch.arange(L - n + lo, L - n + hi, device="cuda")[:, None]
            hide = tok > stand
            if case["window"]:
                hide |= tok <= stand - case["window"]
            for h in range(K):
                score = torch.einsum("tgd,ld->tgl", qs[lo:hi, h], kv[0][:, h]) / math.sqrt(D)
                if case["softcap"]:
                    score = case["softcap"] * torch.tanh(score / case["softcap"])
                score = score.masked_fill(hide[:, None], -math.inf)
                lse[lo:hi, h] = torch.logsumexp(score, -1)
                p = torch.exp(score - lse[lo:hi, h][..., None])
                out[lo:hi, h] = torch.einsum("tgl,ld->tgd", p, kv[1][:, h])
                if case["observe"]:
                    per[:L] += p.sum((0, 1))
        if case["observe"]:
            weight[order[at:at + nb]] += per.view(nb, P).sum(1)
        at += nb
        outs.append(out.reshape(n, K * G, D))
        lses.append(lse.reshape(n, K * G))
    return {"out": torch.cat(outs), "lse": torch.cat(lses), **({"weight": weight} if case["observe"] else {})}
