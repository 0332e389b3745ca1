"""A batch of requests served from one page pool: the host's side of the packed operators.

A step gives every request some more tokens (a whole prompt, a chunk of one, drafts, one token, none), packed row behind row.
`begin` takes their pages from the free list (`vf_pages_assign`), `attend` stores a layer's keys and values and attends over the
cache (`vf_rotary_append`, `vf_attention_packed`), `finish` tells which requests had room: one copy of a few integers, the
step's one synchronisation.  All of them work on the current stream; where it changes, the caller lets the next wait for the last.  `keep` takes back tokens that were not accepted, `release` gives a request's pages back.
The projections around `attend`, the norms and the feed-forward are the caller's.
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
        self.in_step = False

    def _within(self, step, what):
        if self.in_step is not step:
            raise RuntimeError(f"{what} within a step" if self.in_step else f"{what} without a step")

    def begin(self, new):
        """new[b] tokens for request b.  Returns the device's row offsets [n + 1] and the rows' positions (-1: refused).  A step that
        was begun and not finished is given up."""
        self.in_step = False
        if len(new) != len(self.host_lens):
            raise ValueError(f"{len(new)} numbers of tokens for {len(self.host_lens)} requests")
        self.new, rows = [int(w) for w in new], sum(max(0, int(w)) for w in new)
        self.pos = torch.empty(rows, dtype=torch.int32, device=self.device)
        self.slot, self.stream = torch.empty_like(self.pos), vf._stream_of(self.pos)
        # from pinned memory, whose copy nobody waits for; torch keeps the memory until the copy is done
        new_dev = torch.tensor(self.new, dtype=torch.int32, pin_memory=True).to(self.device, non_blocking=True)
        vf.vf_pages_assign(self.lens, new_dev, self.free, self.n_free,
                           self.table, self.row_off, self.pos, self.slot, self.kv_len, self.n_free_after)
        self.workspace, self.max_rows = None, max([0] + self.new)
        self.max_keys = max([0] + [h + w for h, w in zip(self.host_lens, self.new) if w > 0])
        self.in_step = True
        return self.row_off, self.pos

    def attend(self, layer, q, k, v):
        """q [rows, q heads, head_dim], k, v [rows, kv heads, head_dim] before rotation (views of one wider matrix allowed): stores
        k and v, returns the attention of every row, zeros for the rows of a refused request."""
        self._within(True, "attend")
        pool, rotated, out = self.pools[layer], q.new_empty(q.shape), q.new_empty(q.shape)
        vf.vf_rotary_append(q, k, v, self.angles, self.pos, self.slot, rotated, pool, self.pairs)
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

    def keep(self, request, tokens):
        """Of the request's tokens the first `tokens` stay (drafts that were not accepted go); pages behind them are free again.
        Between steps: a step that is open has taken its pages from the free list as it stood."""
        self._within(False, "keep")
        first, last = -(-tokens // PAGE), -(-self.host_lens[request] // PAGE)
        if not 0 <= tokens <= self.host_lens[request]:
            raise ValueError(f"request {request} holds {self.host_lens[request]} tokens, not {tokens}")
        if first < last:
            self.free[self.host_free:self.host_free + last - first] = self.table[request, first:last]
            self.table[request, first:last] = -1
            self.host_free += last - first
            self.n_free.fill_(self.host_free)
        self.lens[request] = tokens
        self.host_lens[request] = tokens

    def release(self, request):
        """The request is over: its place in the batch and its pages are free.  Between steps, as `keep`."""
        self.keep(request, 0)
