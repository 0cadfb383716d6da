"""A serving loop on memory of the pool: what arrives from another function's host memory, and the operators that answer with it.

    python -m paper_2411_01830_amd.serve [--requests 16] [--layers 4] [--steps 32] [--rotate] [--four-bit] [--sample] [--check]

A small transformer of random weights serves requests whose prompts were read elsewhere: their keys and values, and the low-rank
adapters of the models' variants, lie in pinned host memory and are brought into the pool by the transfer engine, a function with
a weight of its own each. Every step drafts a tree of tokens for each request (what followed a token before, and one other token
a level), has the model judge all of them at once, keeps the path that the model would have taken itself, and appends what was
kept to the pages. A request that has its tokens gives its pages back, and another one takes its place.

--rotate gives heads their norms and positions: a row's is that of its level behind the cached tokens. --four-bit keeps the projections' weights in the
pool, in 4 bits, brought by transfers as the adapters are. --sample draws tokens from the model's probabilities instead of taking the likeliest: the drafted
ones are judged by random numbers, so that what is kept is distributed as if each token had been drawn by itself.

--check compares every projection, rotation and attention with plain products over a history kept beside the pages, what is
kept with the definition of judging, and every page's owner after every step.
"""
import argparse
import sys
import time

import numpy as np
import torch

from workloads import DESC_DTYPE, FT_HOST, FT_POOL

from . import binding as ft, harness, operators as ops

SLAB = 64 << 10
CHUNK = 1 << 20
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}    # the roundoff of one rounding


class Server:
    def __init__(self, requests=16, layers=4, hidden=1024, heads=16, kv_heads=4, dim=64, vocab=4096, page=16, prompt=500, answer=40, depth=4,
                 ranks=(8, 16, 32, 12), dtype=torch.bfloat16, check=False, seed=0, rotate=False, four_bit=False, sample=False):
        self.requests, self.layers, self.heads, self.kv_heads, self.dim, self.vocab = requests, layers, heads, kv_heads, dim, vocab
        self.hidden, self.page, self.prompt, self.answer, self.dtype, self.check = hidden, page, prompt, answer, dtype, check
        self.rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)                       # all chance on the GPU: a run is its seed's
        self.random = lambda *shape, by=1.0: (torch.randn(*shape, device="cuda", generator=self.gen) * by).to(dtype)
        self.width = (heads + 2 * kv_heads) * dim
        self.embed = self.random(vocab, hidden)
        self.rotate, self.four_bit, self.sample = rotate, four_bit, sample
        if not four_bit:
            self.w_qkv = [self.random(hidden, self.width, by=hidden ** -0.5) for _ in range(layers)]
            self.w_out = [self.random(heads * dim, hidden, by=(heads * dim) ** -0.5) for _ in range(layers)]

        if not 1 <= depth <= 31:
            raise ValueError("a tree's rows have one word of the mask: 1 to 31 levels")
        # The trees of a step are the same every time: request r drafts 1 + r % depth levels of two tokens below its last one. The first of a
        # level hangs from the first of the level before; row t sees itself and what it hangs from.
        self.levels = [1 + r % depth for r in range(requests)]
        starts, parent, mask, depth_of = [0], [], [], []
        for n in self.levels:
            first, at = len(parent), 0
            parent.append(-1)
            mask.append(1)
            depth_of += [0] + [1 + i // 2 for i in range(2 * n)]
            for _ in range(n):
                here = len(parent) - first
                for k in range(2):
                    parent.append(first + at)
                    mask.append(mask[first + at] | 1 << (here + k))
                at = here
            starts.append(len(parent))
        self.starts_host, self.parent_host, self.mask_host, self.rows = starts, parent, mask, len(parent)
        self.starts, self.parent = self._ints(starts), torch.tensor(parent, device="cuda")
        self.mask = torch.tensor(mask, dtype=torch.int64, device="cuda")
        self.drafts = 1 + 2 * depth
        self.root = self.starts[:-1].long()
        self.deep = [torch.tensor([r for r, n in enumerate(self.levels) if n > level], device="cuda") for level in range(max(self.levels))]
        self.first_of = [self.root[who] + 1 + 2 * level for level, who in enumerate(self.deep)]
        self.level_of = self._ints(depth_of)
        first_of_request = torch.repeat_interleave(torch.tensor(starts[:-1]), torch.tensor(starts).diff())
        self.hangs_from = torch.where(torch.tensor(parent) < 0, -1, torch.tensor(parent) - first_of_request).to(torch.int32).cuda()  # within a request
        self.request_of = torch.repeat_interleave(torch.arange(requests, device="cuda"), torch.tensor(starts, device="cuda").diff())
        self.last = torch.zeros(requests, dtype=torch.int64, device="cuda")               # the token that is to be judged next
        self.follows = torch.zeros(requests, vocab, dtype=torch.int64, device="cuda")     # what followed a token the last time

        # memory of the pool: the cache of every layer, the adapters, and room for one prompt that has arrived and has no pages yet
        self.blocks = -(-(prompt + answer + self.drafts) // page)
        pages = requests * self.blocks
        row = kv_heads * dim * 2
        ranks = list(ranks)
        adapter_bytes = [((hidden + self.width) * r * 2 + SLAB - 1) // SLAB * SLAB for r in ranks]
        cache_bytes = (pages * page * row + SLAB - 1) // SLAB * SLAB
        prompt_bytes = (prompt * row * 2 * layers + SLAB - 1) // SLAB * SLAB
        self.engine = harness.GpuEngine(0)
        weight_bytes = 0
        if four_bit:
            parts = [n for ni, no in ((hidden, self.width), (heads * dim, hidden)) for n in self._parts(ni, no)]
            weight_bytes = layers * sum((n + SLAB - 1) // SLAB * SLAB for n in parts)
        self.engine.pool_create(2 * layers * cache_bytes + layers * (sum(adapter_bytes) + len(ranks) * SLAB) + prompt_bytes + weight_bytes, SLAB, fill=None)
        self.engine.host_arena(max(prompt_bytes, layers * sum(adapter_bytes), weight_bytes), fill=None)
        self.pool = self.engine.pool
        self.memory = self.engine.segments[0][0]
        alloc = self.engine.slab_alloc
        self.caches = [ops.KvCache(self.pool, alloc(cache_bytes), alloc(cache_bytes), pages, page, kv_heads, dim, dtype) for _ in range(layers)]
        self.arrived = alloc(prompt_bytes)
        self.bytes_moved = 0
        self._bring_adapters(ranks, alloc)
        if four_bit:
            self._bring_weights(alloc)
        if rotate:
            self.rotation = ops.Rotation(self.pool, [10000.0 ** (-2 * i / dim) for i in range(dim // 2)], dim)
            self.norms = [(1 + self.random(2, dim, by=0.1)) for _ in range(layers)]

        self.lens = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.table = torch.zeros(requests, self.blocks, dtype=torch.int32, device="cuda")
        self.free = torch.arange(pages, dtype=torch.int32, device="cuda")
        self.state = self._ints([pages, 0, 0, 0])
        self.adapter_of = torch.full((requests,), -1, dtype=torch.int32, device="cuda")
        self.left = np.zeros(requests, dtype=np.int64)                                    # tokens that each request still wants
        self.history = [[None] * requests for _ in range(layers)]
        self.worst = 0.0
        for r in range(requests):
            self._admit(r)

    def _ints(self, values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def _transfer(self, moves, weights):
        """(function, offset in the host arena, offset in the pool, bytes) of each move, in one job."""
        d = np.zeros(len(moves), dtype=DESC_DTYPE)
        for i, (func, src, dst, n) in enumerate(moves):
            d[i]["func"], d[i]["src_space"], d[i]["dst_space"] = func, FT_HOST, FT_POOL
            d[i]["src"], d[i]["dst"], d[i]["row_bytes"], d[i]["rows"] = src, dst, n, 1
        job = self.engine.submit(d, np.asarray(weights, dtype=np.uint32), CHUNK)
        self.engine.wait(job)
        self.bytes_moved += sum(m[3] for m in moves)

    def _host(self, at, n):
        return self.engine.host[at:at + n].view(self.dtype)

    def _bring_adapters(self, ranks, alloc):
        moves, kinds, at = [], [], 0
        for _ in range(self.layers):
            for func, r in enumerate(ranks):
                a, b = r * self.hidden, self.width * r
                self._host(at, 2 * (a + b)).copy_(torch.cat([self.random(a, by=self.hidden ** -0.5), self.random(b, by=r ** -0.5)]))
                to = alloc(2 * (a + b))
                moves.append((func, at, to, 2 * (a + b)))
                kinds.append((to, to + 2 * a, r, 0.5))
                at += (2 * (a + b) + 255) // 256 * 256
        self._transfer(moves, [1] * len(ranks))
        n = len(ranks)
        self.adapters = [ops.Adapters(self.pool, kinds[i * n:i * n + n], self.hidden, self.width, self.dtype) for i in range(self.layers)]
        self.kinds = kinds

    GROUP = 64

    def _parts(self, width_in, width_out):
        """Bytes of a projection's codes, scales and zeros."""
        groups = -(-width_in // self.GROUP)
        return width_out * ((width_in + 1) // 2), 2 * width_out * groups, width_out * groups

    def _bring_weights(self, alloc):
        """Every layer's two projections in 4 bits, random codes from host memory."""
        moves, at, self.w_qkv, self.w_out = [], 0, [], []
        for _ in range(self.layers):
            for ni, no, into in ((self.hidden, self.width, self.w_qkv), (self.heads * self.dim, self.hidden, self.w_out)):
                to = []
                for kind, n in enumerate(self._parts(ni, no)):
                    here = self.engine.host[at:at + n]
                    if kind == 1:                                                 # (codes are 4.6 from their zeros, in the mean of squares)
                        here.view(self.dtype).copy_((torch.rand(n // 2, device="cuda", generator=self.gen) + 0.5).to(self.dtype) * (0.2 * ni ** -0.5))
                    else:
                        here.copy_(torch.randint(256 if kind == 0 else 16, (n,), dtype=torch.uint8, device="cuda", generator=self.gen))
                    to.append(alloc(n))
                    moves.append((0, at, to[-1], n))
                    at += (n + 255) // 256 * 256
                into.append(ops.Linear4(self.pool, to[0], to[1], ni, no, self.GROUP, self.dtype, zeros_off=to[2]))
        self._transfer(moves, [1])

    def _weights(self, w):
        """What a projection's codes stand for, and its factors, in 64 bits."""
        r, groups = w.record, -(-w.width_in // self.GROUP)
        codes = self.memory[r.weights:r.weights + w.width_out * ((w.width_in + 1) // 2)].view(w.width_out, -1)
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(1)[:, :w.width_in].double()
        scales = self.memory[r.scales:r.scales + 2 * w.width_out * groups].view(self.dtype).view(w.width_out, groups)
        zeros = self.memory[r.zeros:r.zeros + w.width_out * groups].view(w.width_out, groups)
        scales, zeros = (t.double().repeat_interleave(self.GROUP, 1)[:, :w.width_in] for t in (scales, zeros))
        return (codes - zeros) * scales, (271 + zeros) * scales

    def _project(self, w, x, base=None):
        if not self.four_bit:
            return x @ w if base is None else base + x @ w
        out = ops.linear4_apply(w, x, base=base)
        if self.check:
            product, terms = self._weights(w)
            want = x.double() @ product.t() + (0 if base is None else base.double())
            # one rounding, and sums in 32 bits of a group's elements whose codes count from a power of two
            slack = 2.0 ** -24 * (self.GROUP + 64) * (x.double().abs() @ terms.t()) + (0 if base is None else 2.0 ** -23 * base.double().abs())
            self._within("projection", out, want.float(), (1.001 * UNIT[self.dtype] * want.abs() + slack).float() + 1e-7)
        return out

    def _adapter(self, layer, i):
        at, b, r, scale = self.kinds[layer * self.adapters[layer].count + i]
        a = self.memory[at:b].view(self.dtype).view(r, self.hidden)
        return a, self.memory[b:b + 2 * self.width * r].view(self.dtype).view(self.width, r), scale

    def _admit(self, r):
        """A request whose prompt's keys and values are in host memory takes place r."""
        n, row = int(self.rng.integers(1, self.prompt + 1)), self.kv_heads * self.dim
        whole = self._host(0, n * row * 2 * 2 * self.layers)
        whole.copy_(self.random(whole.numel()))
        self._transfer([(0, 0, self.arrived, 2 * whole.numel())], [1])
        starts = self._ints([0] * (r + 1) + [n] * (self.requests - r))
        slots, self.lens, self.state = ops.kv_grow(self.pool, self.lens, starts, n, self.table, self.free, self.state, self.page)
        kv = self.memory[self.arrived:self.arrived + 2 * whole.numel()].view(self.dtype).view(self.layers, 2, n, self.kv_heads, self.dim)
        for layer in range(self.layers):
            ops.kv_append(self.caches[layer], kv[layer, 0], kv[layer, 1], slots)
            if self.check:
                self.history[layer][r] = kv[layer].float()
        self.adapter_of[r] = int(self.rng.integers(-1, self.adapters[0].count))
        self.last[r] = int(self.rng.integers(self.vocab))
        self.left[r] = self.answer

    def _draft(self):
        """The tokens of the rows: each request's last one, then what followed it before and one other, level by level."""
        tokens = torch.randint(self.vocab, (self.rows,), device="cuda", generator=self.gen)
        at = self.last
        tokens[self.root] = at
        who = torch.arange(self.requests, device="cuda")
        for level in range(max(self.levels)):
            at = self.follows[who, at]
            tokens[self.first_of[level]] = at[self.deep[level]]
        return tokens

    def _judge(self, tokens, x):
        """Rows that the model would have taken itself; what it takes next."""
        said = (x @ self.embed.t()).argmax(-1)                        # what follows each row

        # a row is kept if the row that it hangs from is, and was followed by its token
        keep = self.parent < 0
        right = ~keep & (said[self.parent.clamp(min=0)] == tokens)
        for level in range(max(self.levels)):
            keep = keep | right & keep[self.parent.clamp(min=0)]
        # of two alike that both hang from the same row the first one stays
        twin = torch.zeros_like(keep)
        twin[1:] = keep[1:] & keep[:-1] & (self.parent[1:] == self.parent[:-1]) & (self.parent[1:] >= 0)
        keep = keep & ~twin
        self.follows[self.request_of[keep], tokens[keep]] = said[keep]
        order = torch.where(keep, torch.arange(self.rows, device="cuda"), -1)
        end = torch.full((self.requests,), -1, device="cuda").scatter_reduce(0, self.request_of, order, "amax")
        self.last = said[end]
        return keep

    def _judge_by_chance(self, tokens, x):
        """Rows that stand against the model's probabilities and random numbers; what was drawn behind them."""
        logits = (x @ self.embed.t()).float()
        target = torch.softmax(logits * (2 / logits.std(-1, keepdim=True)), -1)
        accept, pick = (torch.rand(n, device="cuda", generator=self.gen) for n in (self.rows, self.requests))
        keep, last, token = ops.tree_verify(self.pool, tokens, self.starts, self.drafts, target, accept, pick, parent=self.hangs_from)
        if self.check:
            self._check_judged(tokens, target, accept, pick, keep, last, token)
        hangs = (self.parent >= 0) & (keep != 0)                      # what follows a kept row: its kept child, or what was drawn
        self.follows[self.request_of[hangs], tokens[self.parent[hangs]]] = tokens[hangs]
        self.follows[torch.arange(self.requests, device="cuda"), tokens[last.long()]] = token
        self.last = token
        return keep

    def step(self):
        """One step of all requests: how many tokens each of them got."""
        tokens = self._draft()
        ids = self.adapter_of[self.request_of]
        groups = ops.adapter_groups(self.adapters[0], ids)
        x = self.embed[tokens]
        kept = []
        for layer in range(self.layers):
            base = self._project(self.w_qkv[layer], x)
            qkv = ops.adapters_apply(self.adapters[layer], groups, x, base)
            q, k, v = qkv.view(self.rows, -1, self.dim).split([self.heads, self.kv_heads, self.kv_heads], dim=1)
            if self.rotate:
                positions = self.lens[self.request_of] + self.level_of
                given, norms = (q, k), self.norms[layer]
                q, k = ops.rotate_heads(self.rotation, q, k, positions, q_weight=norms[0], k_weight=norms[1], eps=1e-6)
                if self.check:
                    for x_, y_, w_ in zip(given, (q, k), norms):
                        self._check_rotation(x_, y_, w_, positions)
            o = ops.tree_attention(self.caches[layer], q, k, v, self.starts, self.lens, self.table, self.drafts, self.mask)
            if self.check:
                self._check_projection(layer, ids, x, base, qkv)
                self._check_attention(layer, q, k, v, o)
            kept.append((k, v))
            x = self._project(self.w_out[layer], o.reshape(self.rows, -1), x)
            x = (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(self.dtype)
        keep = self._judge_by_chance(tokens, x) if self.sample else self._judge(tokens, x)

        slots, lens, self.state = ops.kv_grow(self.pool, self.lens, self.starts, self.rows, self.table, self.free, self.state, self.page, keep)
        for layer in range(self.layers):
            ops.kv_append(self.caches[layer], *kept[layer], slots)
            if self.check:
                for r in range(self.requests):
                    mine = torch.arange(self.starts_host[r], self.starts_host[r + 1], device="cuda")
                    mine = mine[keep[mine] != 0]
                    new = torch.stack([kept[layer][0][mine], kept[layer][1][mine]]).float()
                    self.history[layer][r] = torch.cat([self.history[layer][r], new], dim=1)
        got = (lens - self.lens).cpu().numpy()                        # (a wait; choosing by flags, above, is another)
        self.lens = lens
        self.left -= got
        over = self.left <= 0
        if over.any():
            done = torch.tensor(over, device="cuda")
            self.lens, self.state = ops.kv_release(self.pool, done, self.lens, self.table, self.free, self.state, self.page)
            for r in np.flatnonzero(over):
                self._admit(int(r))
        if self.check:
            self._check_pages()
        return got

    # ---- the plain forms -------------------------------------------------------------------------

    def _within(self, what, got, want, bound):
        share = float(((got.float() - want).abs() / bound).max())
        self.worst = max(self.worst, share)
        if not share <= 1:
            raise AssertionError(f"{what}: off by {share:.2f} of what rounding explains")

    def _check_projection(self, layer, ids, x, base, got):
        want, size = base.float(), torch.zeros(self.rows, self.width, device="cuda")
        for i in range(self.adapters[layer].count):
            a, b, scale = self._adapter(layer, i)
            mine = ids == i
            h = x[mine].double() @ a.double().t()
            want[mine] += (scale * (h @ b.double().t())).float()
            size[mine] = (abs(scale) * (h.abs() @ b.double().abs().t())).float()
        self._within("adapters", got, want, UNIT[self.dtype] * want.abs() + 2.0 ** -14 * size + 1e-6)

    def _check_rotation(self, x, got, weight, positions):
        y = x.double()
        y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight.double()
        angle = (positions.double()[:, None] * self.rotation.freqs.double())[:, None]
        a, b = y.split(self.dim // 2, -1)
        want = torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)
        size = (a.abs() + b.abs()).repeat(1, 1, 2)
        self._within("rotation", got, want.float(), (1.001 * UNIT[self.dtype] * want.abs() + 20 * 2.0 ** -24 * size).float() + 1e-7)

    def _check_judged(self, tokens, target, accept, pick, keep, last, token):
        """The definition, row by row, in 64 bits."""
        target, tokens, accept, kept = target.double().cpu(), tokens.tolist(), accept.tolist(), keep.tolist()
        for r in range(self.requests):
            a, b = self.starts_host[r], self.starts_host[r + 1]
            row, stands = a, {a}
            while True:
                left, mass, found = target[row].clone(), 1.0, None
                for t in (t for t in range(row + 1, b) if self.parent_host[t] == row):
                    p = float(left[tokens[t]])
                    if accept[t] * mass < p:
                        found = t
                        break
                    left[tokens[t]], mass = 0, max(mass - p, 0.0)
                if found is None:
                    break
                row = found
                stands.add(row)
            sums = left.cumsum(0)
            drawn = int(torch.nonzero(sums > float(pick[r]) * float(sums[-1]))[0])
            if stands != {t for t in range(a, b) if kept[t]} or int(last[r]) != row or int(token[r]) != drawn:
                raise AssertionError("judged otherwise than the definition says")

    def _check_attention(self, layer, q, k, v, got):
        g = self.heads // self.kv_heads
        for r in range(self.requests):
            a, b = self.starts_host[r], self.starts_host[r + 1]
            keys, values = (torch.cat([self.history[layer][r][i], t[a:b].float()]) for i, t in enumerate((k, v)))
            past = keys.shape[0] - (b - a)
            sees = torch.ones(b - a, keys.shape[0], dtype=torch.bool)
            for i in range(b - a):
                for j in range(b - a):
                    sees[i, past + j] = bool(self.mask_host[a + i] >> j & 1)
            keys, values = (t.transpose(0, 1).repeat_interleave(g, 0).contiguous() for t in (keys, values))
            s = q[a:b].float().transpose(0, 1).contiguous() @ keys.transpose(1, 2).contiguous() * self.dim ** -0.5
            p = s.masked_fill(~sees.to("cuda"), float("-inf")).softmax(-1)
            want = (p @ values).transpose(0, 1)
            size = (p @ values.abs()).transpose(0, 1)                 # a weight is rounded once, and the result
            self._within("attention", got[a:b], want, 2.5 * UNIT[self.dtype] * size + 1e-6)

    def _check_pages(self):
        """Every page is a request's or free, and once."""
        lens, table, free = self.lens.tolist(), self.table.tolist(), self.free.tolist()
        top, lacked, refused, _ = self.state.tolist()
        owned = [p for n, row in zip(lens, table) for p in row[:-(-n // self.page)]]
        if sorted(owned + free[:top]) != list(range(len(free))) or lacked or refused:
            raise AssertionError("pages are lost or owned twice")
        if lens != [h.shape[1] for h in self.history[0]]:
            raise AssertionError("lengths are not those of the history")

    def close(self):
        torch.cuda.synchronize()
        self.engine.close()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--prompt", type=int, default=500, help="the longest prompt, in tokens")
    ap.add_argument("--answer", type=int, default=40, help="the tokens that a request wants")
    ap.add_argument("--depth", type=int, default=4, help="levels of the deepest tree")
    ap.add_argument("--dtype", default="bfloat16", choices=["bfloat16", "float16"])
    ap.add_argument("--rotate", action="store_true", help="norms of heads, and positions")
    ap.add_argument("--four-bit", action="store_true", help="weights of 4 bits, in the pool")
    ap.add_argument("--sample", action="store_true", help="tokens drawn by the model's probabilities")
    ap.add_argument("--check", action="store_true")
    args = ap.parse_args()
    if not torch.cuda.is_available():
        print("needs a GPU", file=sys.stderr)
        sys.exit(2)
    server = Server(args.requests, args.layers, prompt=args.prompt, answer=args.answer, depth=args.depth, dtype=getattr(torch, args.dtype), check=args.check,
                    rotate=args.rotate, four_bit=args.four_bit, sample=args.sample)
    server.step()
    torch.cuda.synchronize()
    begin, tokens = time.perf_counter(), 0
    for _ in range(args.steps):
        tokens += int(server.step().sum())
    torch.cuda.synchronize()
    took = time.perf_counter() - begin
    print(f"{args.steps} steps of {args.requests} requests, {server.rows} rows each: {tokens} tokens, {tokens / args.steps / args.requests:.2f} a request and step, "
          f"{took / args.steps * 1e3:.2f} ms a step; {server.bytes_moved / 1e6:.1f} MB brought from host memory")
    if args.check:
        print(f"every projection, rotation, attention and page checked: at most {server.worst:.2f} of what rounding explains")
    server.close()


if __name__ == "__main__":
    main()
