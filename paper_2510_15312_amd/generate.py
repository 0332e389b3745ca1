"""Greedy generation by repeated draft-verify steps: the host loop around the library's calls.

Every piece of work is a call of the C ABI: chunked prefill (`vf_prefill_chunk`), the retrieval
drafter over the text so far (`vf_draft_suffix_match`), the pool of reusable rejected drafts
(`vf_reuse_pool_*`), the verify forward (`vf_verify`), acceptance (`vf_accept`) and the reuse
segment (`vf_reuse_select`), with `vf_logits_adjust` between the two where the logits are to be adjusted.  This module only strings them together and moves the few integers a
step decides (accepted count, emitted tokens, reuse segment) to the host, once per step.
"""
import numpy as np
import torch

from . import binding as vf


def _best(z):
    """The id of the largest logit as vf_accept has it: the lowest of equal ones, what is not a number never."""
    z = torch.where(z.isnan(), -float("inf"), z)
    return int((z == z.max()).nonzero()[0])


def _sent(numbers, dev):
    """On the device, from pinned memory, whose copy nobody waits for; torch keeps the memory until the copy is done."""
    return torch.tensor(numbers, dtype=torch.int32, pin_memory=True).to(dev, non_blocking=True)


class _Adjust:
    """What `generate` puts on the logits: the text so far on the device, biases, and the masks of a step's rows."""

    def __init__(self, penalties, biases, allowed, prompt, room, vocab, dev):
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
        self.allowed, self.vocab, self.dev, self.ints = allowed, vocab, dev, ints
        self.logits = torch.empty((vf.VF_MAX_DRAFTS + 1, vocab), dtype=torch.float32, device=dev)
        self.more = {}
        if penalties is not None:
            penalties = list(penalties)
            as_held = torch.tensor(penalties, dtype=torch.float32).tolist()      # (1e50 is infinite, 1e-50 zero)
            if len(penalties) != 3 or not 0 < as_held[0] < float("inf") or as_held[1] + as_held[2] != as_held[1] + as_held[2]:
                raise ValueError(f"penalties {penalties}: a finite repetition above 0, presence, frequency")
            self.more = dict(penalties=torch.tensor([penalties], dtype=torch.float32, device=dev), prompt_len=ints([len(prompt)]),
                             history=torch.zeros((1, room), dtype=torch.int32, device=dev), history_len=ints([0]))
        if biases:
            if any(value != value for value in biases.values()):
                raise ValueError(f"biases that are not numbers: {biases}")
            self.more["biases"] = (ints([0, len(biases)]), ints(list(biases)), torch.tensor(list(biases.values()), dtype=torch.float32, device=dev))
        self.length = 0

    def admitted(self, text, drafts):
        """The drafts in front of the first that its row's ids exclude, none of which could be accepted: `allowed` is asked about
        texts that it admits only.  Keeps the masks of their rows."""
        self.mask = None
        if self.allowed is None:
            return drafts
        bits, rows = np.zeros((len(drafts) + 1, -(-self.vocab // 32) * 32), bool), []
        for i in range(len(drafts) + 1):
            ids = self.allowed(list(text) + list(drafts[:i]))
            rows.append(-1 if ids is None else i)
            if ids is None:
                continue
            ids = [int(v) for v in ids]
            if not all(0 <= v < self.vocab for v in ids):
                raise ValueError(f"allowed ids outside the vocabulary of {self.vocab}")
            bits[i, ids] = True
            if i < len(drafts) and not (0 <= drafts[i] < self.vocab and bits[i, drafts[i]]):
                drafts = drafts[:i]
                break
        self.mask = np.packbits(bits[:len(rows)], axis=1, bitorder="little").view(np.int32), rows
        return drafts

    def prepare(self, text, tokens, drafts):
        """Sends what the rows of the text's end and of the drafts behind it need, ahead of the forward pass, so that nothing waits for that.
        tokens: the rows' tokens on the device; the first of them, the pending token, counts as the end of the text."""
        self.rows, self.args = len(drafts) + 1, dict(self.more, row_off=_sent([0, len(drafts) + 1], self.dev))
        if "history" in self.more:
            self.args["history"][0, self.length:len(text)] = _sent(text[self.length:], self.dev)
            self.args["history_len"].fill_(len(text))
            self.length = len(text)
            self.args["tokens"] = tokens
        if self.mask is not None:
            words, rows = self.mask
            self.args.update(mask=torch.from_numpy(words).pin_memory().to(self.dev, non_blocking=True), mask_row=_sent(rows, self.dev))

    def __call__(self):
        """The logits of the prepared rows, in place."""
        logits = self.logits[:self.rows]
        vf.vf_logits_adjust(logits, out=logits, **self.args)
        return logits


def generate(model, seq, prompt, n_new, k=16, max_suffix=8, min_suffix=1, chunk=256, reuse_max_age=2, drafter=None, reuse=True,
             penalties=None, biases=None, allowed=None):
    """prompt: host ints, none where the sequence has its pending token already; returns (the n_new generated tokens, statistics).  Greedy acceptance: the
    result is what plain greedy decoding would produce.  drafter(text, k) -> list of at most k draft
    ids replaces the library's suffix-match drafter (any drafter gives the same text); reuse=False
    leaves the pool of rejected drafts out.

    The logits are adjusted before a token is taken from them (`vf_logits_adjust`), so that the text is what plain greedy
    decoding with the same adjustments would produce: penalties (a finite repetition above 0, presence, frequency); biases {id: value};
    allowed(text) -> the ids that may follow a text, prompt included, or None for all.  `allowed` is asked about the text so far and about
    what it admits behind it, no other drafts; drafts that it excludes are not verified.  Where it allows no id, 0 follows, as in any
    row that is all -infinity."""
    dev = model.buf.device
    k = min(int(k), vf.VF_MAX_DRAFTS)
    toks = torch.as_tensor(list(prompt), dtype=torch.int32, device=dev)
    adjust = None
    if penalties is not None or biases or allowed is not None:
        adjust = _Adjust(penalties, biases, allowed, prompt, len(prompt) + n_new + vf.VF_MAX_DRAFTS + 1, model.cfg.vocab, dev)
    for c0 in range(0, len(prompt), chunk):
        last = c0 + chunk >= len(prompt)
        vf.vf_prefill_chunk(model, seq, toks[c0:c0 + chunk], sample_first=last, logits_mode=int(last and adjust is not None),
                            logits_out=adjust.logits if last and adjust is not None else None)
    length, pending = vf.vf_seq_get_state(seq)
    if adjust is not None and len(prompt):              # the first token comes from adjusted logits too
        adjust.admitted([int(t) for t in prompt], [])
        adjust.prepare([int(t) for t in prompt], None, [])
        pending = _best(adjust()[0])
        vf.vf_seq_set_pending(seq, pending)
    text = [int(t) for t in prompt] + [pending]        # the pending token is the first generated one
    pool = vf.vf_reuse_pool_init(reuse_max_age, max(k, 1))
    n_acc = torch.zeros(1, dtype=torch.int32, device=dev)
    out = torch.zeros(vf.VF_MAX_DRAFTS + 1, dtype=torch.int32, device=dev)
    y = torch.zeros_like(out)
    seg = torch.zeros(2, dtype=torch.int32, device=dev)
    greedy = [(vf.VF_GREEDY, 0.0, None, None)]
    steps, accepted, drafted = 0, 0, 0
    while len(text) - len(prompt) < n_new:
        if not k:
            fresh = []
        elif drafter is not None:
            fresh = [int(t) for t in drafter(text, k)][:k]
        else:
            fresh = vf.vf_draft_suffix_match(text, k, max_suffix, min_suffix)
        proposed = vf.vf_reuse_pool_extend(pool, fresh) if k and reuse else fresh
        drafts = proposed if adjust is None else adjust.admitted(text, proposed)
        m = len(drafts) + 1
        tokens = _sent([vf.VF_PENDING] + drafts, dev)
        logits = None
        if adjust is None:
            vf.vf_verify(model, [seq], tokens, [0, m])
        else:
            adjust.prepare(text, tokens, drafts)
            vf.vf_verify(model, [seq], tokens, [0, m], adjust.logits)
            logits = adjust()
        vf.vf_accept(model, [seq], tokens, [0, m], greedy, n_acc, out[:m], y[:m], logits)
        if drafts and reuse:
            vf.vf_reuse_select(tokens, [0, m], y[:m], n_acc, seg)
        host = torch.cat([n_acc, seg, out[:m]]).cpu().tolist()          # the step's one synchronisation
        a, seg_start, seg_len, emitted = host[0], host[1], host[2], host[3:4 + host[0]]
        if proposed and reuse:      # (a pool whose drafts are all excluded ages too)
            vf.vf_reuse_pool_update(pool, drafts, *((seg_start, seg_len) if drafts else (0, 0)))
        text += emitted
        length += 1 + a
        vf.vf_seq_note_len(seq, length)                 # vf_accept counted all m rows; 1 + a were kept
        steps += 1
        accepted += a
        drafted += len(drafts)
    new = text[len(prompt):len(prompt) + n_new]
    return new, {"steps": steps, "accepted_drafts": accepted, "drafted": drafted,
                 "tokens_per_step": (len(text) - len(prompt) - 1) / max(steps, 1)}
