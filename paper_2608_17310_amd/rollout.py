"""Scoring a member: a dense decoder evaluated over the parameters that a plan
moves (Section 3 of arXiv 2608.17310: apply, evaluate, revert).

    plan = esopt.Plan(params)                    # workloads.decoder_shapes order
    model = Decoder(params, q_heads=32, kv_heads=8, head_dim=128, tied=True,
                    seqs=32, length=2048, format="e4m3")
    run_generation(plan, seeds, signs, sigma, alpha,
                   evaluate=lambda i: reward(model.generate(prompts, 64)))

The decoder reads the parameters in place, so it always evaluates the member that
is applied.  Queries and keys are normalised for each head, rotated and stored
by KVCache.append, and attended to by KVCache.attend; matrix products and the
elementwise rest are PyTorch's.  One pool of pages serves all layers: layer l
takes the pages l * pages_per_layer and on.

Prompts of any lengths are packed without padding.  After `prefill` every
`step` appends one token to each sequence.

Rewards: `log_likelihood` through logits rounded to bf16, a slab of rows at a time;
`score`, the same sum from logits in 32 bits that are never stored; `divergence`, the
distance from a teacher's `top_logits`.  With `adapters` each sequence is
evaluated under its own member's low-rank adapters (`assign`), a whole
population in one batch.
"""

import torch
import torch.nn.functional as F

from .head import Head
from .kvcache import KVCache

# Logits that log_likelihood holds at once (in bf16 and float32, and their
# log-softmax: 10 bytes each).
LOGITS_AT_A_TIME = 1 << 28

# Rows that `score` and `divergence` take to the head at once, at most: its calls have up to
# 65536, and 2^36 logits.
ROWS_AT_A_TIME = 1 << 15

PROJECTIONS = ("q", "k", "v", "o", "gate", "up", "down")


def rope_table(positions, rot, base=10000.0, device="cuda"):
    """Cosines and sines of the rotation, [positions, rot] float32, from 64 bits."""
    freq = base ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


class Decoder:
    """A decoder over `params`, bf16 tensors in the order of
    workloads.decoder_shapes (embedding; per layer q, k, v, o, gate, up, down
    and two norms; final norm; head unless tied).  `seqs` sequences of up to
    `length` tokens share the cache.  q_gains and k_gains ([layers, head_dim]
    bf16) are the gains of the head norms (None: ones).  cap: the cap of the
    attention scores.  adapters: for each layer a dict of adapters.Adapters by
    projection ("q", "k", "v", "o", "gate", "up", "down"; those not in it have
    none), or None."""

    def __init__(self, params, q_heads, kv_heads, head_dim, tied, seqs, length, format="e4m3",
                 page=64, rope_base=10000.0, eps=1e-6, q_gains=None, k_gains=None, cap=0.0,
                 adapters=None):
        params = list(params)
        per_layer = 9
        body = len(params) - (2 if tied else 3)
        if body < 0 or body % per_layer:
            raise ValueError("params are not in the order of workloads.decoder_shapes")
        self.embedding = params[0]
        self.layers = [params[1 + per_layer * i:1 + per_layer * (i + 1)]
                       for i in range(body // per_layer)]
        self.final_norm = params[1 + body]
        self.head = self.embedding if tied else params[2 + body]
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.eps, self.cap, self.page, self.length = eps, cap, page, length
        dev = self.embedding.device
        n = len(self.layers)
        if adapters is not None and len(adapters) != n:
            raise ValueError(f"adapters for {len(adapters)} layers of {n}")
        for layer in adapters or ():
            if not set(layer) <= set(PROJECTIONS):
                raise ValueError(f"adapters must be named {', '.join(PROJECTIONS)}, got "
                                 f"{', '.join(map(str, layer))}")
        self.adapters = adapters
        self.members = torch.full((seqs,), -1, dtype=torch.int32, device=dev)
        ones = torch.ones(n, head_dim, dtype=torch.bfloat16, device=dev)
        self.q_gains = ones if q_gains is None else q_gains
        self.k_gains = ones if k_gains is None else k_gains
        self.rope = rope_table(length, head_dim, rope_base, dev)
        per_seq = -(-length // page)
        self.pages_per_layer = seqs * per_seq
        self.cache = KVCache.allocate(n * self.pages_per_layer, kv_heads, head_dim, format, page, dev)
        self.tables = [torch.arange(i * self.pages_per_layer, (i + 1) * self.pages_per_layer,
                                    dtype=torch.int32, device=dev).view(seqs, per_seq)
                       for i in range(n)]
        self.lengths = torch.zeros(seqs, dtype=torch.int32, device=dev)
        self.longest = 0                        # the host's bound of the lengths
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.member_status = torch.zeros(1, dtype=torch.int32, device=dev)   # ES_ADAPT_BAD_INDEX

    def _norm(self, x, gain):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + self.eps) * gain.float()).to(x.dtype)

    def _check_ids(self, tokens):
        """Refuse token ids outside the vocabulary, which would index past the embedding."""
        low, high = (int(x) for x in tokens.aminmax())
        if low < 0 or high >= len(self.embedding):
            raise ValueError(f"token ids must lie in [0, {len(self.embedding)}), got {low} .. {high}")

    def assign(self, members):
        """The member whose adapters each sequence is evaluated under, [seqs]
        (negative: none).  What is already in the cache stays as it is.  Numbers
        on the GPU are not read back to be checked."""
        members = torch.as_tensor(members)
        if members.is_floating_point():
            raise ValueError(f"members must be integers, not {members.dtype}")
        if members.shape != self.members.shape:
            raise ValueError(f"members of shape {tuple(members.shape)} for {len(self.members)} sequences")
        if self.adapters is None:
            raise ValueError("the decoder has no adapters")
        least = min((a.members for layer in self.adapters for a in layer.values()), default=0)
        if not members.is_cuda and len(members) and int(members.max()) >= least:
            raise ValueError(f"members must be below {least}, got {int(members.max())}")
        self.members.copy_(members.long().clamp(-1, 2 ** 31 - 1))   # (what int32 cannot hold is no member)

    def _forward(self, tokens, seq, positions, starts, max_rows):
        """Hidden states [tokens, hidden] of packed tokens, whose keys and values
        are appended; self.lengths already counts them."""
        hq, h, d = self.q_heads, self.kv_heads, self.head_dim
        member = None if self.adapters is None else self.members[seq]

        def project(y, w, layer, name):
            a = None if member is None else self.adapters[layer].get(name)
            return F.linear(y, w) if a is None else a.project(y, w, member, status=self.member_status)

        place = (self.tables[0][seq, positions // self.page].long() * self.page
                 + positions % self.page)
        x = self.embedding[tokens]
        positions = positions.int()
        for i, (wq, wk, wv, wo, gate, up, down, norm1, norm2) in enumerate(self.layers):
            y = self._norm(x, norm1)
            q = self.cache.append(project(y, wk, i, "k").view(-1, h, d),
                                  project(y, wv, i, "v").view(-1, h, d),
                                  place + i * self.pages_per_layer * self.page,
                                  q=project(y, wq, i, "q").view(-1, hq, d), q_gain=self.q_gains[i],
                                  k_gain=self.k_gains[i], eps=self.eps, rope=self.rope,
                                  positions=positions, status=self.status)
            a = self.cache.attend(q, self.tables[i], self.lengths, starts, max_rows=max_rows,
                                  max_length=self.longest, cap=self.cap, status=self.status)
            x = x + project(a.view(-1, hq * d), wo, i, "o")
            y = self._norm(x, norm2)
            x = x + project(F.silu(project(y, gate, i, "gate")) * project(y, up, i, "up"), down, i, "down")
        return self._norm(x, self.final_norm)

    def _pack(self, prompts):
        if len(prompts) != len(self.lengths):
            raise ValueError(f"{len(prompts)} prompts for {len(self.lengths)} sequences")
        sizes = [len(p) for p in prompts]
        if min(sizes) < 1 or max(sizes) > self.length:
            raise ValueError(f"prompts must have 1 .. {self.length} tokens")
        dev = self.embedding.device
        tokens = torch.cat([torch.as_tensor(p, dtype=torch.long) for p in prompts])
        self._check_ids(tokens)
        tokens = tokens.to(dev)
        n = torch.tensor(sizes, dtype=torch.int32)
        starts = torch.cat([torch.zeros(1, dtype=torch.int32), n.cumsum(0, dtype=torch.int32)])
        seq = torch.repeat_interleave(torch.arange(len(sizes)), n)
        positions = torch.arange(len(seq)) - starts[:-1].long()[seq]
        self.lengths.copy_(n)
        self.longest = max(sizes)
        return tokens, seq.to(dev), positions.to(dev), starts.to(dev), sizes

    def prefill(self, prompts):
        """Logits [seqs, vocabulary] (float32) after each prompt; the cache holds
        the prompts."""
        tokens, seq, positions, starts, sizes = self._pack(prompts)
        x = self._forward(tokens, seq, positions, starts, max(sizes))
        return F.linear(x[starts[1:].long() - 1], self.head).float()

    def step(self, tokens):
        """Append one token to each sequence; logits [seqs, vocabulary] (float32).
        Ids on the GPU are not read back to be checked."""
        tokens = torch.as_tensor(tokens, dtype=torch.long)
        if tokens.shape != self.lengths.shape:
            raise ValueError(f"tokens of shape {tuple(tokens.shape)} for {len(self.lengths)} sequences")
        if self.longest >= self.length:
            raise ValueError(f"sequences have at most {self.length} tokens")
        if not tokens.is_cuda:
            self._check_ids(tokens)
        dev = self.embedding.device
        positions = self.lengths.long()
        self.lengths += 1
        self.longest += 1
        rows = torch.arange(len(tokens) + 1, dtype=torch.int32, device=dev)
        x = self._forward(tokens.to(dev), rows[:-1].long(), positions, rows, 1)
        return F.linear(x, self.head).float()

    def generate(self, prompts, count):
        """`count` greedy tokens after each prompt, [seqs, count] (ties: the lowest)."""
        if count < 0:
            raise ValueError(f"count must not be negative, got {count}")
        logits = self.prefill(prompts)
        out = torch.empty(len(logits), count, dtype=torch.long, device=logits.device)
        for i in range(count):
            out[:, i] = logits.argmax(-1)
            if i + 1 < count:
                logits = self.step(out[:, i])
        return out

    def _answers(self, prompts, targets):
        """The rows that predict the targets' tokens: hidden states of all tokens, the
        rows' numbers, the tokens after them, and where each belongs: (sequence,
        place in its target), of [seqs, longest target]."""
        prompts, targets = list(map(list, prompts)), list(map(list, targets))
        if len(prompts) != len(targets):
            raise ValueError(f"{len(prompts)} prompts for {len(targets)} targets")
        if not all(prompts):
            raise ValueError("prompts must have at least one token")
        whole = [p + t for p, t in zip(prompts, targets)]
        tokens, seq, positions, starts, sizes = self._pack(whole)
        x = self._forward(tokens, seq, positions, starts, max(sizes))
        begin = torch.tensor([len(p) for p in prompts], device=tokens.device)
        # row r predicts token r + 1; rows from the prompt's last on, but the sequence's last
        size = (starts[1:] - starts[:-1]).long()
        rows = torch.nonzero((positions >= begin[seq] - 1) & (positions + 1 < size[seq])).flatten()
        at = seq[rows], positions[rows] + 1 - begin[seq[rows]]
        return x, rows, tokens[rows + 1], at, (len(sizes), max(map(len, targets)))

    def _slabs(self, rows):
        slab = min(ROWS_AT_A_TIME, (1 << 36) // len(self.head))
        return ((i, i + slab) for i in range(0, rows, slab))

    @staticmethod
    def _sums(terms, at, shape):
        """The sum of each sequence's terms, in one order: rewards are the same every time."""
        room = torch.zeros(shape, dtype=torch.float64, device=terms.device)
        room[at] = terms.double()
        return room.sum(1).float()

    def log_likelihood(self, prompts, targets):
        """Sum of the log-probabilities of each target's tokens after its prompt,
        [seqs] (float32): the usual reward of a supervised task.  Prompts have at
        least one token: a sequence's first is predicted by nothing."""
        x, rows, tokens, at, shape = self._answers(prompts, targets)
        got = torch.empty(len(rows), dtype=torch.float32, device=rows.device)
        slab = max(1, LOGITS_AT_A_TIME // len(self.head))
        for i in range(0, len(rows), slab):
            logp = F.linear(x[rows[i:i + slab]], self.head).float().log_softmax(-1)
            got[i:i + slab] = logp.gather(1, tokens[i:i + slab, None])[:, 0]
        return self._sums(got, at, shape)

    def score(self, prompts, targets):
        """log_likelihood, [seqs] (float32), from logits in 32 bits, which are not
        stored: nearer to the model's own by the logits' rounding to bf16."""
        x, rows, tokens, at, shape = self._answers(prompts, targets)
        got = torch.empty(len(rows), dtype=torch.float32, device=rows.device)
        for i, j in self._slabs(len(rows)):
            got[i:j] = Head(self.head).score(x[rows[i:j]], tokens[i:j])[0]
        return self._sums(got, at, shape)

    def top_logits(self, prompts, targets, count):
        """The `count` largest logits (float32) and their tokens (int64), [rows, count],
        in front of each of the targets' tokens, the targets one after another:
        what `divergence` of another model takes."""
        x, rows, _, _, _ = self._answers(prompts, targets)
        ids = torch.empty(len(rows), count, dtype=torch.long, device=rows.device)
        logits = torch.empty(len(rows), count, dtype=torch.float32, device=rows.device)
        slab = max(1, LOGITS_AT_A_TIME // len(self.head))
        for i in range(0, len(rows), slab):
            # not rounded to bf16 on the way: `divergence` has the student's in 32 bits too
            logits[i:i + slab], ids[i:i + slab] = torch.mm(
                x[rows[i:i + slab]], self.head.t(), out_dtype=torch.float32).topk(count, -1)
        return ids, logits

    def divergence(self, prompts, targets, ids, logits, scale=1.0):
        """Sum over each target's tokens of the divergence from a teacher, [seqs]
        (float32): its logits [rows, entries] (float32) at ids [rows, entries]
        (int64; negative: none) in front of each of the targets' tokens, the
        targets one after another.  Its negative is a reward.  scale: the
        inverse temperature."""
        if ids.dim() != 2 or logits.shape != ids.shape:
            raise ValueError("ids and logits must be [rows, entries]")
        targets = list(map(list, targets))
        if len(ids) != sum(map(len, targets)):
            raise ValueError(f"a teacher's {len(ids)} rows for {sum(map(len, targets))} tokens")
        x, rows, _, at, shape = self._answers(prompts, targets)
        got = torch.empty(len(rows), dtype=torch.float32, device=rows.device)
        for i, j in self._slabs(len(rows)):
            got[i:j] = Head(self.head).distill(x[rows[i:j]], ids[i:j], logits[i:j], scale=scale)[0]
        return self._sums(got, at, shape)
