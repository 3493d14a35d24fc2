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
"""

import torch
import torch.nn.functional as F

from .kvcache import KVCache

# Logits that log_likelihood holds at once (in bf16 and float32, and their
# log-softmax: 10 bytes each).
LOGITS_AT_A_TIME = 1 << 28


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
    attention scores."""

    def __init__(self, params, q_heads, kv_heads, head_dim, tied, seqs, length, format="e4m3",
                 page=64, rope_base=10000.0, eps=1e-6, q_gains=None, k_gains=None, cap=0.0):
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

    def _norm(self, x, gain):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + self.eps) * gain.float()).to(x.dtype)

    def _check_ids(self, tokens):
        """Refuse token ids outside the vocabulary, which would index past the embedding."""
        low, high = (int(x) for x in tokens.aminmax())
        if low < 0 or high >= len(self.embedding):
            raise ValueError(f"token ids must lie in [0, {len(self.embedding)}), got {low} .. {high}")

    def _forward(self, tokens, seq, positions, starts, max_rows):
        """Hidden states [tokens, hidden] of packed tokens, whose keys and values
        are appended; self.lengths already counts them."""
        hq, h, d = self.q_heads, self.kv_heads, self.head_dim
        place = (self.tables[0][seq, positions // self.page].long() * self.page
                 + positions % self.page)
        x = self.embedding[tokens]
        positions = positions.int()
        for i, (wq, wk, wv, wo, gate, up, down, norm1, norm2) in enumerate(self.layers):
            y = self._norm(x, norm1)
            q = self.cache.append(F.linear(y, wk).view(-1, h, d), F.linear(y, wv).view(-1, h, d),
                                  place + i * self.pages_per_layer * self.page,
                                  q=F.linear(y, wq).view(-1, hq, d), q_gain=self.q_gains[i],
                                  k_gain=self.k_gains[i], eps=self.eps, rope=self.rope,
                                  positions=positions, status=self.status)
            a = self.cache.attend(q, self.tables[i], self.lengths, starts, max_rows=max_rows,
                                  max_length=self.longest, cap=self.cap, status=self.status)
            x = x + F.linear(a.view(-1, hq * d), wo)
            y = self._norm(x, norm2)
            x = x + F.linear(F.silu(F.linear(y, gate)) * F.linear(y, up), down)
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

    def log_likelihood(self, prompts, targets):
        """Sum of the log-probabilities of each target's tokens after its prompt,
        [seqs] (float32): the usual reward of a supervised task.  Prompts have at
        least one token: a sequence's first is predicted by nothing."""
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
        got = torch.empty(len(rows), dtype=torch.float32, device=rows.device)
        slab = max(1, LOGITS_AT_A_TIME // len(self.head))
        for i in range(0, len(rows), slab):
            r = rows[i:i + slab]
            logp = F.linear(x[r], self.head).float().log_softmax(-1)
            got[i:i + slab] = logp.gather(1, tokens[r + 1][:, None])[:, 0]
        # a row for each sequence, summed in one order: rewards are the same every time
        terms = torch.zeros(len(sizes), max(map(len, targets)), dtype=torch.float64, device=got.device)
        terms[seq[rows], positions[rows] + 1 - begin[seq[rows]]] = got.double()
        return terms.sum(1).float()
