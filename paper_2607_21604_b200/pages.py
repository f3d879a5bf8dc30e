"""The host's account of a paged 4-bit cache: which pages belong to which sequence.

`PagePool` owns the pages of all layers and the page numbers of sequences; the library's kernels read and write
what is in them.  Sequences that branch share their pages; the last, half-filled one is copied when a branch grows.
All copies are enqueued on the current stream, before the calls that use the pages.
"""
from __future__ import annotations

import torch

from . import binding
from .binding import PAGE_TOKENS, AkvsError


class PagePool:
    def __init__(self, n_layers, n_pages, n_kv, hd, device="cuda"):
        nbytes = binding.page_bytes(n_kv, hd)
        if nbytes < 0 or n_layers < 0 or n_pages < 0:
            raise AkvsError(-1, "PagePool")
        self.pool = torch.zeros((n_layers, n_pages, nbytes), dtype=torch.uint8, device=device)
        self.users = [0] * n_pages                    # sequences that hold a page
        self.free = list(range(n_pages - 1, -1, -1))  # the lowest number is taken first
        self.pages, self.length, self._next = {}, {}, 0

    def __getitem__(self, layer):
        """The pool of one layer, as op_pages_append and op_attention_pages take it."""
        return self.pool[layer]

    def open(self):
        """A new, empty sequence."""
        s, self._next = self._next, self._next + 1
        self.pages[s], self.length[s] = [], 0
        return s

    def grow(self, seqs, n=1):
        """Room for n more tokens (a number, or one per sequence) in each of `seqs`, which become part of their
        lengths.  A last page that others hold too is copied first.  Raises, and changes nothing, where pages run out or a
        copy is refused."""
        seqs = list(seqs)
        ns = [n] * len(seqs) if isinstance(n, int) else list(n)
        if len(ns) != len(seqs) or len(set(seqs)) != len(seqs) or any(x < 0 for x in ns):
            raise AkvsError(-1, "PagePool.grow")
        plan, left = [], {}
        for s, x in zip(seqs, ns):
            have, length = self.pages[s], self.length[s]
            shared = x > 0 and length % PAGE_TOKENS != 0 and left.setdefault(have[-1], self.users[have[-1]]) > 1
            if shared:
                left[have[-1]] -= 1                   # the last of those that branch keeps the page
            plan.append((s, x, shared, -(-(length + x) // PAGE_TOKENS) - len(have)))
        need = sum(more + shared for _, _, shared, more in plan)
        if need > len(self.free):
            raise AkvsError(-8, "PagePool.grow")
        # The copies first: where one is refused, the account is as it was.
        taken, src, dst = self.free[len(self.free) - need:], [], []       # the last is taken first
        pages = {}
        for s, x, shared, more in plan:
            pages[s] = list(self.pages[s])
            if shared:
                src.append(pages[s][-1])
                pages[s][-1] = taken.pop()
                dst.append(pages[s][-1])
            pages[s] += [taken.pop() for _ in range(more)]
        self._copy(src, dst)
        del self.free[len(self.free) - need:]
        for s, x, shared, more in plan:
            for page in pages[s][len(pages[s]) - more - shared:]:
                self.users[page] = 1
            self.pages[s] = pages[s]
            self.length[s] += x
        for page in src:
            self.users[page] -= 1

    def fork(self, seq, n=1):
        """n sequences that go on from where `seq` is; all of them share what it holds."""
        new, pages, length = [], self.pages[seq], self.length[seq]
        for _ in range(n):
            s = self.open()
            self.pages[s], self.length[s] = list(pages), length
            for page in pages:
                self.users[page] += 1
            new.append(s)
        return new

    def cut(self, seq, length):
        """Forgets the tokens of `seq` from `length` on."""
        if not 0 <= length <= self.length[seq]:
            raise AkvsError(-1, "PagePool.cut")
        keep = -(-length // PAGE_TOKENS)
        self._drop(self.pages[seq][keep:])
        self.pages[seq], self.length[seq] = self.pages[seq][:keep], length

    def close(self, seq):
        """Ends a sequence; pages that nobody else holds are free again."""
        self._drop(self.pages.pop(seq))
        del self.length[seq]

    def compact(self):
        """Moves the pages in use to the lowest numbers and returns how many moved: the pages from there on may be given
        back.  Tables made before are void."""
        used = sum(1 for u in self.users if u)
        src = [p for p in range(used, len(self.users)) if self.users[p]]
        dst = [p for p in range(used) if not self.users[p]]
        to = dict(zip(src, dst))
        self._copy(src, dst)
        for a, b in to.items():
            self.users[a], self.users[b] = 0, self.users[a]
        for s, pages in self.pages.items():
            self.pages[s] = [to.get(p, p) for p in pages]
        self.free = list(range(len(self.users) - 1, used - 1, -1))
        return len(src)

    def table(self, seqs):
        """(table [S][width], lens [S]) of these sequences on the pool's device."""
        seqs = list(seqs)
        width = max((len(self.pages[s]) for s in seqs), default=0)
        rows = [self.pages[s] + [-1] * (width - len(self.pages[s])) for s in seqs]
        table = torch.tensor(rows, dtype=torch.int32).reshape(len(seqs), width)
        lens = torch.tensor([self.length[s] for s in seqs], dtype=torch.int32)
        return table.to(self.pool.device), lens.to(self.pool.device)

    def _drop(self, pages):
        for page in pages:
            self.users[page] -= 1
            if not self.users[page]:
                self.free.append(page)

    def _copy(self, src, dst):
        step = 65535                                  # pairs of a call
        for i in range(0, len(src), step):
            a, b = (torch.tensor(x[i:i + step], dtype=torch.int32).to(self.pool.device) for x in (src, dst))
            binding.op_pages_copy(self.pool, a, b)
