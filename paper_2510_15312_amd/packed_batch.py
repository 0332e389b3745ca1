"""A batch of requests served from one page pool: the host's side of the packed operators.

A step gives every request some more tokens (a whole prompt, a chunk of one, drafts, one token, none), packed row behind row.
`begin` takes their pages from the free list (`vf_pages_assign`), `attend` stores a layer's keys and values and attends over the
cache (`vf_rotary_append`, `vf_attention_packed`), `finish` tells which requests had room: one copy of a few integers, the
step's one synchronisation.  All of them work on the current stream; where it changes, the caller lets the next wait for the last.  `keep` takes back tokens that were not accepted, `release` gives a request's pages back.
Requests may branch: `fork` lets a place that holds nothing go on from another request's text, whose full pages the two then share
(`vf_pages_fork`), `keep_all` cuts or ends many at once (`vf_pages_keep`), `compact` moves everything to a pool of another size
(`vf_pages_compact`).  `adjust` puts penalties, biases and masks on a step's logits (`vf_logits_adjust`).
The projections around `attend`, the norms of whole rows and the feed-forward are the caller's.
"""
import torch

from . import binding as vf

PAGE = 64


class PackedBatch:
    def __init__(self, n_requests, n_layers, n_q_heads, n_kv_heads, head_dim, pool_pages, max_tokens, dtype=torch.bfloat16,
                 rotary_dim=None, theta=1e6, pairs=vf.VF_ROTARY_HALF, device="cuda:0"):
        """Room for n_requests requests of at most max_tokens tokens each, in pool_pages pages of 64 tokens together."""
        def ints(*shape, value=0):
            return torch.full(shape, value, dtype=torch.int32, device=device)
        self.heads, self.pairs, self.device = (n_q_heads, n_kv_heads, head_dim), pairs, device
        self.max_pages = -(-max_tokens // PAGE)
        self.pools = torch.zeros((n_layers, pool_pages, 2, n_kv_heads, PAGE * head_dim), dtype=dtype, device=device)
        self.angles = vf.vf_rotary_table(rotary_dim or head_dim, theta, PAGE * self.max_pages, device=device)
        self.table = ints(n_requests, self.max_pages, value=-1)
        self.free = torch.arange(pool_pages, dtype=torch.int32, device=device)
        self.n_free, self.n_free_after = ints(1, value=pool_pages), ints(1)
        self.lens, self.row_off, self.kv_len = ints(n_requests), ints(n_requests + 1), ints(n_requests)
        self.host_lens, self.host_free = [0] * n_requests, pool_pages
        self.shares, self.copies, self.n_copies = ints(pool_pages), ints(n_requests, 2), ints(1)
        self.shared = False             # whether a page may have several holders
        self.in_step = False

    def _within(self, step, what):
        if self.in_step is not step:
            raise RuntimeError(f"{what} within a step" if self.in_step else f"{what} without a step")

    def _sent(self, numbers):
        """On the device, from pinned memory, whose copy nobody waits for; torch keeps the memory until the copy is done."""
        return torch.tensor(numbers, dtype=torch.int32, pin_memory=True).to(self.device, non_blocking=True)

    def begin(self, new):
        """new[b] tokens for request b.  Returns the device's row offsets [n + 1] and the rows' positions (-1: refused).  A step that
        was begun and not finished is given up."""
        self.in_step = False
        if len(new) != len(self.host_lens):
            raise ValueError(f"{len(new)} numbers of tokens for {len(self.host_lens)} requests")
        self.new, rows = [int(w) for w in new], sum(max(0, int(w)) for w in new)
        self.pos = torch.empty(rows, dtype=torch.int32, device=self.device)
        self.slot, self.stream = torch.empty_like(self.pos), vf._stream_of(self.pos)
        vf.vf_pages_assign(self.lens, self._sent(self.new), self.free, self.n_free,
                           self.table, self.row_off, self.pos, self.slot, self.kv_len, self.n_free_after)
        self.workspace, self.max_rows = None, max([0] + self.new)
        self.max_keys = max([0] + [h + w for h, w in zip(self.host_lens, self.new) if w > 0])
        self.in_step = True
        return self.row_off, self.pos

    def attend(self, layer, q, k, v, norms=None):
        """q [rows, q heads, head_dim], k, v [rows, kv heads, head_dim] before rotation (views of one wider matrix allowed): stores
        k and v, returns the attention of every row, zeros for the rows of a refused request.  norms: (gains of q, gains of k, eps) of
        a model that normalises its heads (`vf_norm_rotary_append`)."""
        self._within(True, "attend")
        pool, rotated, out = self.pools[layer], q.new_empty(q.shape), q.new_empty(q.shape)
        if norms is None:
            vf.vf_rotary_append(q, k, v, self.angles, self.pos, self.slot, rotated, pool, self.pairs)
        else:
            vf.vf_norm_rotary_append(q, k, v, *norms, self.angles, self.pos, self.slot, rotated, pool, self.pairs)
        stream = vf._stream_of(q)
        if stream != self.stream:       # another than begin's
            self.pos.record_stream(torch.cuda.current_stream(self.device))
            self.slot.record_stream(torch.cuda.current_stream(self.device))
        if self.workspace is None:      # the layers of a step share it
            self.workspace = vf.vf_attention_packed_workspace(rotated, pool, self.table, self.max_rows, self.max_keys)
            self.workspace_stream = stream
        elif stream != self.workspace_stream:
            self.workspace.record_stream(torch.cuda.current_stream(self.device))
        vf.vf_attention_packed(rotated, pool, self.table, self.row_off, self.kv_len, out, self.max_rows, self.max_keys, self.workspace)
        return out

    def adjust(self, logits, tokens=None, out=None, **more):
        """The step's logits [rows, vocab] with penalties, biases and masks, in float32: `vf_logits_adjust` with the step's rows.
        tokens int32 [rows]: the rows' tokens, where they count and the history does not have them yet; out: logits itself is allowed."""
        self._within(True, "adjust")
        out = torch.empty(logits.shape, dtype=torch.float32, device=logits.device) if out is None else out
        vf.vf_logits_adjust(logits, self.row_off, out, tokens=tokens, **more)
        return out

    def finish(self):
        """Ends the step: the lengths move on, the free list is what is left.  Returns a truth value per request: False where
        the pool or the table had no room, so that the request stands as before and may ask again."""
        self._within(True, "finish")
        self.in_step = False
        torch.where(self.kv_len > 0, self.kv_len, self.lens, out=self.lens)
        self.n_free, self.n_free_after = self.n_free_after, self.n_free
        *lens, self.host_free = torch.cat([self.kv_len, self.n_free]).tolist()
        granted = [length > 0 or w == 0 for length, w in zip(lens, self.new)]
        self.host_lens = [length or before for length, before in zip(lens, self.host_lens)]
        return granted

    def _moved_on(self):
        """Lengths and free list as a call between steps has left them, on the device and, by one copy, on the host."""
        self.lens.copy_(self.kv_len)
        self.n_free, self.n_free_after = self.n_free_after, self.n_free
        *self.host_lens, self.host_free = torch.cat([self.lens, self.n_free]).tolist()

    def fork(self, sources, targets, tokens=None):
        """Request targets[i], which holds nothing, goes on from the first tokens[i] tokens of request sources[i] (default: all that
        it holds): the full pages are shared, of the last one it gets a copy.  Between steps, as `keep`.  Returns a truth value per fork:
        False where the pool had no page for the copy, so that the target still holds nothing."""
        self._within(False, "fork")
        n, held = len(self.host_lens), self.host_lens
        sources, targets = [int(x) for x in sources], [int(x) for x in targets]
        if not all(0 <= x < n for x in sources + targets):
            raise ValueError(f"requests {sources} and {targets} of {n}")
        tokens = [held[x] for x in sources] if tokens is None else [int(x) for x in tokens]
        if not len(sources) == len(targets) == len(tokens):
            raise ValueError(f"{len(sources)} sources, {len(targets)} targets, {len(tokens)} numbers of tokens")
        if len(set(targets)) < len(targets) or any(held[x] for x in targets):
            raise ValueError(f"targets {targets} hold tokens, or one is named twice")
        if not all(0 <= t <= held[x] for t, x in zip(tokens, sources)):
            raise ValueError(f"requests {sources} hold {[held[x] for x in sources]} tokens, not {tokens}")
        if not sources:
            return []
        src, dst, take = self._sent([sources, targets, tokens])
        vf.vf_pages_fork(src, dst, take, self.lens, self.free, self.n_free, self.table, self.shares, self.kv_len, self.n_free_after,
                         self.copies, self.n_copies)
        self.shared = True
        vf.vf_pages_copy(self.pools, self.copies, self.n_copies, self.pools)
        self._moved_on()
        return [self.host_lens[x] == t for x, t in zip(targets, tokens)]

    def keep_all(self, tokens):
        """Of every request b the first tokens[b] tokens stay (None: all); pages that nobody holds any more are free again.  A
        request that is cut inside a page that others hold gets a copy of it; where the pool has none left it keeps its full pages only.
        Between steps, as `keep`.  Returns what the requests hold now."""
        self._within(False, "keep_all")
        held = self.host_lens
        if len(tokens) != len(held):
            raise ValueError(f"{len(tokens)} numbers of tokens for {len(held)} requests")
        tokens = [-1 if t is None else int(t) for t in tokens]
        if not all(-1 <= t <= h for t, h in zip(tokens, held)):
            raise ValueError(f"requests hold {held} tokens, not {tokens}")
        vf.vf_pages_keep(self.lens, self._sent(tokens), self.free, self.n_free, self.table, self.shares, self.kv_len, self.n_free_after,
                         self.copies, self.n_copies)
        if self.shared:                 # else no page has two holders
            vf.vf_pages_copy(self.pools, self.copies, self.n_copies, self.pools)
        self._moved_on()
        self.shared = self.shared and any(self.host_lens)
        return list(self.host_lens)

    def compact(self, pool_pages):
        """Moves all requests to a pool of pool_pages pages, of which they take the first ones.  Between steps, as `keep`."""
        self._within(False, "compact")
        pages = self.free.numel()
        if pool_pages < max(1, pages - self.host_free):
            raise ValueError(f"the requests hold {pages - self.host_free} pages, more than {pool_pages}")
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=self.device)  # noqa: E731
        pools = self.pools.new_zeros((self.pools.shape[0], pool_pages, *self.pools.shape[2:]))
        shares, free, moved, copies = ints(pool_pages), ints(pool_pages), ints(pages), ints(min(pages, pool_pages), 2)
        vf.vf_pages_compact(self.lens, self.table, self.shares, self.table, shares, free, self.n_free, moved, copies, self.n_copies)
        vf.vf_pages_copy(self.pools, copies, self.n_copies, pools)
        for old in (self.pools, self.shares, self.free):
            old.record_stream(torch.cuda.current_stream(self.device))
        self.pools, self.shares, self.free = pools, shares, free
        self.host_free += pool_pages - pages

    def keep(self, request, tokens):
        """Of the request's tokens the first `tokens` stay (drafts that were not accepted go); pages behind them are free again.
        Between steps: a step that is open has taken its pages from the free list as it stood.  Returns what the request holds now."""
        self._within(False, "keep")
        request = range(len(self.host_lens))[request]       # (-1: the last)
        first, last = -(-tokens // PAGE), -(-self.host_lens[request] // PAGE)
        if not 0 <= tokens <= self.host_lens[request]:
            raise ValueError(f"request {request} holds {self.host_lens[request]} tokens, not {tokens}")
        if self.shared:
            return self.keep_all([tokens if b == request else None for b in range(len(self.host_lens))])[request]
        if first < last:                # pages with one holder: the host knows what becomes of them, and nobody waits
            self.free[self.host_free:self.host_free + last - first] = self.table[request, first:last]
            self.table[request, first:last] = -1
            self.host_free += last - first
            self.n_free.fill_(self.host_free)
        self.lens[request] = tokens
        self.host_lens[request] = tokens
        return tokens

    def release(self, request):
        """The request is over: its place in the batch and its pages are free.  Between steps, as `keep`."""
        self.keep(request, 0)
