"""Performance cases of the paged key-value cache: appending to it and attention over it.

A pool of pages ([pages][kv heads][page tokens][head dim], one array for K and one for V) holds
the tokens of many sequences; a table names each sequence's pages.

  append   K (and Q) of the new tokens rotated by their positions, K and V written to the pages
  attend   attention of the new tokens over the pages of their sequences: one new token each
           (decoding), a few, or a whole prompt or renderer chunk

listed() names a fixed set, draw() gives more of the same ranges; prepare() makes what a program
holds before the call, run() is one pass (plain torch operations, or with `own` the framework's
kernels), work() the bytes and operations it cannot do without, exact() the same outputs in
float64.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List, Optional, Tuple

import torch

own = False

THETA = 10000.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name: Optional[str], kind: str, dtype: str, q_heads: int, kv_heads: int, d: int, page: int,
          seqs: int, new: Tuple[int, int], past: Tuple[int, int], block: bool = False,
          window: int = -1, anchors: int = 0, grid_w: int = 0, grid_h: int = 0, pad: int = 0) -> Dict:
    """new, past: fewest and most new and earlier tokens of a sequence; grid_h x grid_w tokens per
    video frame (0: text, whose position is the index in the sequence); pad: rows behind the last
    sequence, as a program with fixed-size buffers has them."""
    c = dict(kind=kind, dtype=dtype, q_heads=q_heads, kv_heads=kv_heads, head_dim=d, page=page,
             seqs=seqs, new_lo=new[0], new_hi=new[1], past_lo=past[0], past_hi=past[1], block=block,
             window=window, anchors=anchors, grid_h=grid_h, grid_w=grid_w, pad=pad)
    return dict(name=name, **c) if name else c


def listed() -> List[Dict]:
    return [
        # one new token of one conversation: the smallest call, all latency
        _case("append_1_token", "append", "bf16", 32, 8, 128, 16, 1, (1, 1), (700, 700)),
        # a decoding step of a full server batch: 200 sequences of every age, padded to 256 rows
        _case("append_200_tokens", "append", "bf16", 32, 8, 128, 16, 200, (1, 1), (1, 400), pad=56),
        # one layer's 14B 480p renderer chunk, three frames of 30 x 52 tokens at their own positions
        _case("append_14b_480p_chunk", "append", "bf16", 40, 40, 128, 64, 1, (4680, 4680), (4680, 4680),
              grid_h=30, grid_w=52),
        # prompts of a small model in float32, ragged
        _case("append_prompts_f32_d64", "append", "f32", 12, 4, 64, 32, 5, (37, 611), (0, 90)),
        # one conversation just begun, small model: the smallest attention call
        _case("decode_1_short_d64", "attend", "bf16", 8, 2, 64, 16, 1, (1, 1), (332, 332)),
        # one conversation over a long document: few rows, a long axis
        _case("decode_1_long", "attend", "bf16", 32, 8, 128, 16, 1, (1, 1), (32773, 32773)),
        # a decoding step of a server batch, ragged lengths: the most bytes
        _case("decode_64_ragged", "attend", "bf16", 32, 8, 128, 16, 64, (1, 1), (150, 12000)),
        # the same kind of step in float32 with a head of its own per query head, a validation run
        _case("decode_16_f32", "attend", "f32", 12, 12, 128, 32, 16, (1, 1), (60, 2300)),
        # a few proposed tokens per stream checked at once, over the first tokens and a window
        _case("verify_4_tokens_window", "attend", "bf16", 40, 8, 128, 32, 12, (2, 5), (900, 9000),
              window=2047, anchors=64),
        # two prompts, causal: the most operations
        _case("prompt_2_causal", "attend", "bf16", 32, 8, 128, 16, 2, (3700, 5003), (0, 300)),
        # a renderer chunk of a preview clip (three frames of 15 x 26) as one bidirectional block over
        # four earlier chunks and three anchor frames, 1.3B heads
        _case("chunk_1.3b_15x26", "attend", "bf16", 12, 12, 128, 64, 1, (1170, 1170), (9360, 9360),
              block=True, window=4680, anchors=1170, grid_h=15, grid_w=26),
        # a slice of a long prompt beside decoding sequences in one call
        _case("mixed_slice_and_decode", "attend", "bf16", 32, 8, 128, 16, 12, (1, 512), (100, 4000)),
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> Dict:
    top = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in top), max(w["flops"] for w in top)
    while True:
        kind = rng.choice(["append", "decode", "decode", "few", "prompt", "chunk"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        d = rng.choice([64, 128, 128])
        kv = rng.choice([1, 2, 3, 4, 5, 8, 8, 12])
        group = rng.choice([1, 1, 2, 3, 4, 4, 5, 7, 8, 16])
        page = rng.choice([16, 16, 32, 64, 128, 256])
        window = rng.choice([-1, -1, -1, _log_int(rng, 1, 4000)])
        anchors = rng.choice([0, 1, 4, 100, 390]) if window >= 0 else 0
        past = _log_int(rng, 1, 32768)
        low = rng.choice([0, past // 20, past])
        if kind == "append":
            seqs = _log_int(rng, 1, 256)
            new = _log_int(rng, 1, 4680)
            c = _case(None, "append", dtype, kv * group, kv, d, page, seqs, (rng.choice([0, 1, new]), new),
                      (0, min(past, 2000)), grid_h=rng.choice([0, 30]), grid_w=52,
                      pad=rng.choice([0, 0, 9]))
        elif kind == "decode":
            c = _case(None, "attend", dtype, kv * group, kv, d, page, _log_int(rng, 1, 256), (1, 1),
                      (low, past), window=window, anchors=anchors, pad=rng.choice([0, 0, 7]))
        elif kind == "few":
            c = _case(None, "attend", dtype, kv * group, kv, d, page, _log_int(rng, 1, 48),
                      (rng.choice([0, 1, 2]), rng.randint(2, 17)), (low, past), window=window,
                      anchors=anchors)
        elif kind == "prompt":
            c = _case(None, "attend", dtype, kv * group, kv, d, page, rng.randint(1, 8),
                      (1, _log_int(rng, 20, 5000)), (0, min(past, 6000)), window=window, anchors=anchors)
        else:
            gh, gw = rng.randint(6, 30), rng.randint(8, 52)
            c = _case(None, "attend", dtype, kv, kv, d, page, rng.randint(1, 2), (3 * gh * gw, 3 * gh * gw),
                      (3 * gh * gw * rng.randint(0, 4),) * 2, block=True, window=3 * gh * gw * rng.randint(0, 4),
                      anchors=gh * gw * rng.randint(0, 3), grid_h=gh, grid_w=gw)
        w = work(c)
        heavy = 0.1 if dtype == "f32" else 1.0    # the float32 matrix rate is a tenth of the bf16 one
        if (0 < w["bytes"] <= most_bytes and w["flops"] <= heavy * most_flops
                and _padded(c) <= 2 ** 32 and _pool_bytes(c) <= 2 ** (29 if kind == "append" else 31)):
            return c


# ---- sizes -------------------------------------------------------------------------
def _lengths(c: Dict) -> List[Tuple[int, int]]:
    """(new tokens, tokens with them) of each sequence: fixed by the case; the first sequence has
    the most of both, the others lie in between, evenly or nearer to the fewest."""
    rng = random.Random(c["seqs"] * 7919 + c["past_hi"] * 31 + c["new_hi"])
    out = []
    for s in range(c["seqs"]):
        new = c["new_hi"] if s == 0 else int(c["new_lo"] + (c["new_hi"] - c["new_lo"]) * rng.random() ** 3)
        past = c["past_hi"] if s == 0 else int(c["past_lo"] + (c["past_hi"] - c["past_lo"]) * rng.random() ** 1.5)
        out.append((new, past + new))
    return out


def _columns(c: Dict) -> int:
    return max(1, max((length + c["page"] - 1) // c["page"] for _, length in _lengths(c)))


def _padded(c: Dict) -> int:
    """Scores of the batch padded to its longest sequence."""
    lens = _lengths(c)
    if c["kind"] == "append":
        return 0
    return c["seqs"] * c["q_heads"] * max(n for n, _ in lens) * max(length for _, length in lens)


def _pool_bytes(c: Dict) -> int:
    size = 2 if c["dtype"] == "bf16" else 4
    pages = sum((length + c["page"] - 1) // c["page"] for _, length in _lengths(c)) + 3
    return pages * c["page"] * c["kv_heads"] * c["head_dim"] * size


def _seen(c: Dict, new: int, length: int) -> Tuple[int, int]:
    """(query-key pairs, keys that any query sees) of one sequence."""
    w, a = c["window"], c["anchors"]
    if new == 0:
        return 0, 0
    first = length - new
    if w < 0:
        return (new * length if c["block"] else sum(range(first + 1, length + 1))), length
    if c["block"]:
        low = max(0, first - w)
        keys = length - low + min(a, low)
        return new * keys, keys
    pairs = sum(min(i, w) + 1 + min(a, max(0, i - w)) for i in range(first, length))
    low = max(0, first - w)
    return pairs, length - low + min(a, low)


def work(c: Dict) -> Dict:
    size = 2 if c["dtype"] == "bf16" else 4
    d, hq, hk = c["head_dim"], c["q_heads"], c["kv_heads"]
    lens = _lengths(c)
    tokens = sum(n for n, _ in lens)
    if c["kind"] == "append":
        return {"bytes": float(2 * tokens * (hq + 2 * hk) * d * size + (12 * tokens if c["grid_h"] else 0)),
                "flops": float(3 * tokens * (hq + hk) * d)}
    seen = [_seen(c, n, length) for n, length in lens]
    return {"bytes": float(sum(k for _, k in seen) * 2 * hk * d * size + 2 * tokens * hq * d * size),
            "flops": float(sum(p for p, _ in seen) * 4 * d * hq)}


# ---- inputs ------------------------------------------------------------------------
def prepare(c: Dict, seed: int) -> Dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = DTYPES[c["dtype"]]
    d, hq, hk, page = c["head_dim"], c["q_heads"], c["kv_heads"], c["page"]
    lens = _lengths(c)
    tokens = sum(n for n, _ in lens)
    rows = tokens + c["pad"]
    columns = _columns(c)
    used = [(length + page - 1) // page for _, length in lens]
    n_pages = sum(used) + 3

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    # pages in any order, as a pool hands them out over time; what no sequence holds is stale
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((c["seqs"], columns), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(used):
        table[s, :n] = order[at:at + n]
        at += n
    starts = torch.tensor([0] + [n for n, _ in lens], dtype=torch.int64).cumsum(0)
    s: Dict = {
        "case": c, "q_start": starts.to(torch.int32).cuda(),
        "kv_len": torch.tensor([length for _, length in lens], dtype=torch.int32, device="cuda"),
        "page_table": table.cuda(), "max_new": max(n for n, _ in lens), "min_new": min(n for n, _ in lens),
        "k_pages": normal(n_pages, hk, page, d), "v_pages": normal(n_pages, hk, page, d),
    }
    if c["kind"] == "append":
        # Q, K and V as one projection writes them, side by side in a row per token
        s["qkv"] = normal(rows, hq + 2 * hk, d)
        s["q_out"] = torch.zeros((rows, hq, d), dtype=dt, device="cuda")
        s["positions"] = _video_positions(c, lens, rows).cuda() if c["grid_h"] else None
    else:
        s["q"] = normal(rows, hq, d)
        s["out"] = torch.zeros_like(s["q"])
    return s


def _video_positions(c: Dict, lens: List[Tuple[int, int]], rows: int) -> torch.Tensor:
    """(frame, row, column) of each new token of a clip."""
    index = torch.cat([torch.arange(length - n, length) for n, length in lens])
    index = torch.cat([index, torch.zeros(rows - index.numel(), dtype=index.dtype)])
    g = c["grid_h"] * c["grid_w"]
    return torch.stack([index // g, index % g // c["grid_w"], index % c["grid_w"]], 1).to(torch.int32)


# ---- one pass ----------------------------------------------------------------------
def run(s: Dict):
    if s["case"]["kind"] == "append":
        return _append(s)
    return _attend(s)


def _split(d: int) -> Tuple[int, int, int]:
    """Rotation pairs of the t, h and w axes."""
    return d // 2 - 2 * (d // 6), d // 6, d // 6


def _append(s: Dict):
    c = s["case"]
    hq, hk = c["q_heads"], c["kv_heads"]
    q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hk], s["qkv"][:, hq + hk:]
    if own:
        from paper_2609_32540_amd import ff

        ff.paged_append(k, v, s["k_pages"], s["v_pages"], s["q_start"], s["kv_len"], s["page_table"],
                        q=q, q_out=s["q_out"], positions=s["positions"])
    else:
        seq, index = _tokens(s)
        n = seq.numel()
        pos = s["positions"][:n] if s["positions"] is not None else index[:, None].expand(n, 3)
        page = s["page_table"][seq, index // c["page"]].long()
        slot = index % c["page"]
        s["k_pages"][page, :, slot] = _rotate(k[:n], pos)
        s["v_pages"][page, :, slot] = v[:n]
        s["q_out"][:n] = _rotate(q[:n], pos)
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _tokens(s: Dict):
    """Sequence and index in it of every new token."""
    start = s["q_start"].long()
    counts = start[1:] - start[:-1]
    n = sum(n for n, _ in _lengths(s["case"]))
    seq = torch.repeat_interleave(torch.arange(counts.numel(), device=start.device), counts, output_size=n)
    index = torch.arange(n, device=start.device) - start[seq] + (s["kv_len"].long() - counts)[seq]
    return seq, index


def _rotate(x: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
    angles = torch.cat([pos[:, a:a + 1].double() * THETA ** (-torch.arange(m, device=x.device, dtype=torch.float64) / m)
                        for a, m in enumerate(_split(x.shape[-1]))], 1)[:, None]
    cos, sin = angles.cos(), angles.sin()
    a, b = x[..., 0::2].double(), x[..., 1::2].double()
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2).to(x.dtype)


def _attend(s: Dict):
    c = s["case"]
    if own:
        from paper_2609_32540_amd import ff

        return ff.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["q_start"], s["kv_len"], s["page_table"],
                                  block=c["block"], window=c["window"], anchor_tokens=c["anchors"],
                                  min_new=s["min_new"], max_new=s["max_new"], out=s["out"])
    d, hk, group, page = c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["page"]
    n_seqs, new = c["seqs"], s["max_new"]
    if new == 0:
        return s["out"]
    dev = s["q"].device
    # keys and values of every sequence in order, padded to the longest
    pages = s["page_table"].long().clamp(min=0)
    keys = pages.shape[1] * page
    k = s["k_pages"][pages].transpose(1, 2).reshape(n_seqs, hk, keys, d).float()
    v = s["v_pages"][pages].transpose(1, 2).reshape(n_seqs, hk, keys, d).float()
    # queries padded to the most new tokens
    start, length = s["q_start"].long(), s["kv_len"].long()
    count = start[1:] - start[:-1]
    tau = torch.arange(new, device=dev)
    row = (start[:-1, None] + tau).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float().reshape(n_seqs, new, hk, group, d).permute(0, 2, 1, 3, 4).reshape(n_seqs, hk, new * group, d)
    # what each new token sees
    j = torch.arange(keys, device=dev)
    first = (length - count)[:, None]
    high = length[:, None].expand(n_seqs, new) if c["block"] else first + tau + 1
    see = j < high[..., None]
    if c["window"] >= 0:
        low = (first.expand(n_seqs, new) if c["block"] else first + tau) - c["window"]
        see = see & ((j >= low[..., None]) | (j < c["anchors"]))
    see = see[:, None, :, None].expand(n_seqs, 1, new, group, keys).reshape(n_seqs, 1, new * group, keys)
    p = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).masked_fill_(~see, -math.inf)
    p = p.sub_(p.amax(3, keepdim=True).clamp(min=-1e30)).exp_()
    total = p.sum(3, keepdim=True)
    o = (p @ v) / total.clamp(min=1e-30)
    o = o.reshape(n_seqs, hk, new, group, d).permute(0, 2, 1, 3, 4).reshape(n_seqs, new, hk * group, d)
    seq, index = _tokens(s)
    s["out"][:seq.numel()] = o[seq, index - first[seq, 0]].to(s["q"].dtype)
    return s["out"]


# ---- float64 -----------------------------------------------------------------------
def exact(c: Dict, seed: int):
    s = prepare(c, seed)
    if c["kind"] == "append":
        return _append64(s)
    return _attend64(s)


def _append64(s: Dict):
    c = s["case"]
    hq, hk, page, d = c["q_heads"], c["kv_heads"], c["page"], c["head_dim"]
    x = s["qkv"].double()
    turn = torch.zeros((x.shape[0], d // 2), dtype=torch.float64, device=x.device)
    where, begin = [], 0
    table = s["page_table"].cpu()
    for n_s, (n, length) in enumerate(_lengths(c)):
        index = torch.arange(length - n, length)
        if s["positions"] is not None:
            pos = s["positions"][begin:begin + n].cpu()
        else:
            pos = index[:, None].repeat(1, 3)
        pair = 0
        for axis, m in enumerate(_split(d)):
            for j in range(m):
                turn[begin:begin + n, pair] = (pos[:, axis].double() * math.pow(THETA, -j / m)).to(x.device)
                pair += 1
        where.append(table[n_s, index // page].long() * page + index % page)
        begin += n
    at = torch.cat(where).to(x.device)
    z = torch.view_as_complex(x[:, :hq + hk].reshape(x.shape[0], hq + hk, d // 2, 2).contiguous())
    z = torch.view_as_real(z * torch.polar(torch.ones_like(turn), turn)[:, None]).flatten(2)
    pools = []
    for pool, new in ((s["k_pages"], z[:begin, hq:]), (s["v_pages"], x[:begin, hq + hk:])):
        flat = pool.double().transpose(1, 2).reshape(-1, hk, d)     # by token slot
        flat[at] = new
        pools.append(flat.reshape(pool.shape[0], page, hk, d).transpose(1, 2))
    q = z[:, :hq].clone()
    q[begin:] = 0
    return {"q": q, "k_pages": pools[0], "v_pages": pools[1]}


def _attend64(s: Dict):
    c = s["case"]
    d, hk, group, page = c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["page"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["q"].device)
    table, begin = s["page_table"].cpu(), 0
    for n_s, (n, length) in enumerate(_lengths(c)):
        pages = [int(p) for p in table[n_s, :(length + page - 1) // page]]
        if n == 0:
            continue
        j = torch.arange(length, device=out.device)
        i = torch.arange(length - n, length, device=out.device)[:, None]
        gone = torch.zeros((n, length), dtype=torch.bool, device=out.device) if c["block"] else j > i
        if c["window"] >= 0:
            since = torch.full_like(i, length - n) if c["block"] else i
            gone = gone | ((j < since - c["window"]) & (j >= c["anchors"]))
        for h in range(hk):
            k = torch.cat([s["k_pages"][p, h] for p in pages])[:length].double()
            v = torch.cat([s["v_pages"][p, h] for p in pages])[:length].double()
            for e in range(h * group, (h + 1) * group):
                x = (s["q"][begin:begin + n, e].double() @ k.T) / math.sqrt(d)
                out[begin:begin + n, e] = torch.softmax(x.masked_fill_(gone, -math.inf), 1) @ v
        begin += n
    return out
