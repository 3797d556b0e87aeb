"""Asynchronous decoding over the 8-bit or 4-bit paged cache: the operators together, as a model's forward pass calls them.

A Session owns the device buffers of a batch of requests and, on the host, which thread of a request sees which.  Rows carry the
tag of the thread that wrote them; a thread is the set of tags that it sees.  A fork gives both the child and the parent a new tag: the child goes on from
what its parent saw then, and does not see what the parent writes later.  A join adds a thread's set to another's.  When a request's last but one thread
has joined, everything written so far becomes a prefix that all of its rows see, and its tags are free again.

A step is begin() with the threads that write a row, then layer() for every layer; nothing in it depends on values on the device, so a step of the same
threads can be captured into a graph and replayed, each replay one token further (run this file for an example).  Between replays other steps may be
begun, of other requests too; the captured one keeps its own rows, for which see again().

With rope, layer() turns q and k by the rows' position ids on their way.  With vocab, a step's rows may be drafts: verify() holds them to the target's
probabilities, and the next begin() or again() takes back those that were not accepted, in a replayed graph as well.  settle() tells the host how far it went.
"""
from __future__ import annotations

from collections import Counter
from dataclasses import dataclass, field

import torch

from . import kv4, kv8, rows

TAGS = 64


@dataclass
class Thread:
    request: int
    tag: int
    sees: int  # set of tags
    position: int = 0  # of its next row
    alive: bool = True


@dataclass
class _Request:
    threads: list = field(default_factory=list)
    used: int = 0  # set of tags


class Session:
    cache = None  # the handle of the 4-bit cache; the 8-bit cache's does everything itself
    places = places_workspace = None  # configuration and workspace of the handle that gives places to the 4-bit cache's rows
    rows_cfg = rows_workspace = rows = keep = None  # of rope and drafts
    _unsettled = False  # threads do not know their positions

    def __init__(self, *, codes="e4m3", dtype="bf16", n_q_heads, n_kv_heads, head_dim, softmax_scale, n_layers=1, max_requests=1, max_rows=256,
                 page_tokens=16, n_phys_pages, pages_per_request, slopes=None, logit_cap=0.0, rope=None, vocab=0, device="cuda:0"):
        """`codes`: e4m3, int8 or e2m1 (4 bits).  `rope`: arguments of rows.make_config that begin with rope_.  `vocab`: of drafts that are to be verified."""
        self.device = torch.device(device)
        sizes = dict(n_layers=n_layers, max_requests=max_requests, max_rows=max_rows, page_tokens=page_tokens, n_phys_pages=n_phys_pages,
                     pages_per_request=pages_per_request)
        i32, u8 = dict(dtype=torch.int32, device=self.device), dict(dtype=torch.uint8, device=self.device)
        # codes and scales are uninitialised on purpose: what has not been written is never read
        if codes == "e2m1":
            self.cfg = cfg = kv4.make_config(dtype, n_q_heads, n_kv_heads, head_dim, softmax_scale, **sizes)
            self.k_codes, self.v_codes, self.k_scale, self.v_scale = (torch.empty(s, **u8) for s in kv4.cache_shapes(cfg))
            # (places go by none of an attention's sizes: the least there are, since the workspace holds a plan's partial rows, too, which nobody asks for)
            self.places = kv8.make_config("e4m3", dtype, 1, 1, 64, 1.0, **{**sizes, "n_layers": 1})
            self.places_workspace = torch.empty(kv8.query_workspace_bytes(self.places), **u8)
        else:
            self.cfg = cfg = kv8.make_config(codes, dtype, n_q_heads, n_kv_heads, head_dim, softmax_scale, **sizes)
            k_shape, v_shape, s_shape = kv8.cache_shapes(cfg)
            self.k_codes, self.v_codes = torch.empty(k_shape, **u8), torch.empty(v_shape, **u8)
            self.k_scale, self.v_scale = torch.empty(s_shape, device=self.device), torch.empty(s_shape, device=self.device)
        if rope is not None or vocab:
            turns = {}
            if rope is not None:
                td = {kv8.BF16: torch.bfloat16, kv8.F16: torch.float16}[cfg.dtype]
                self._q, self._k = (torch.empty(max_rows, h, head_dim, dtype=td, device=self.device) for h in (n_q_heads, n_kv_heads))
                f = torch.as_tensor(rope["rope_frequency"], dtype=torch.float64).to(self.device)
                turns = dict(n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, **{**rope, "rope_frequency": f})
            self.rows_cfg = rows.make_config(max_rows=max_rows, vocab=vocab, max_sequences=max_requests if vocab else 0, **turns)
            self.rows_workspace = torch.empty(rows.query_workspace_bytes(self.rows_cfg), **u8)
        if vocab:
            # how much of every request the next step keeps: its length, but for what verify() writes.  (Replays write it unseen by the host, so every step
            # goes by it, and leaves it as one that is not verified would.)
            self.keep, self._no_rows = torch.zeros(max_requests, **i32), torch.zeros(max_requests + 1, **i32)
            self.accepted, self.next_token = torch.zeros(max_requests, **i32), torch.full((max_requests,), -1, **i32)
        self.page_table = torch.full((max_requests, pages_per_request), -1, **i32)
        self.free_pages = torch.arange(n_phys_pages - 1, -1, -1, **i32)
        self.free_count = torch.full((1,), n_phys_pages, **i32)
        self.length = torch.zeros(max_requests, **i32)
        self.prefix_len = torch.zeros(max_requests, **i32)
        slots = n_phys_pages * page_tokens
        self.slot_tag, self.slot_position = torch.zeros(slots, dtype=torch.uint8, device=self.device), torch.zeros(slots, **i32)
        self.slot = torch.full((max_rows,), -1, **i32)
        self.workspace = torch.empty((kv4 if codes == "e2m1" else kv8).query_workspace_bytes(cfg), **u8)
        self.slopes = None if slopes is None else torch.as_tensor(slopes, dtype=torch.float32, device=self.device)
        self.logit_cap = logit_cap
        self.requests = [_Request() for _ in range(max_requests)]
        self.handle = self._step = self._stream = None
        self._captured = []  # steps that graphs read: their memory stays the session's
        self.bind(torch.cuda.current_stream(self.device))

    def bind(self, stream):
        """Work of later calls goes to this stream; the caller orders it behind what was enqueued before.  A step that had begun goes on with again()."""
        self._stream = stream
        shared = dict(page_table=self.page_table, slot_tag=self.slot_tag, slot_position=self.slot_position, stream=stream.cuda_stream)
        held = dict(k_codes=self.k_codes, v_codes=self.v_codes, k_scale=self.k_scale, v_scale=self.v_scale)
        if self.places is not None:
            self.handle = kv8.PastaKv8(self.places, self.places_workspace, free_pages=self.free_pages, **shared)
            self.cache = kv4.PastaKv4(self.cfg, self.workspace, **held, **shared)
        else:
            self.handle = kv8.PastaKv8(self.cfg, self.workspace, free_pages=self.free_pages, **held, **shared)
        if self.rows_cfg is not None:
            self.rows = rows.PastaRows(self.rows_cfg, self.rows_workspace, stream=stream.cuda_stream)
        if self._step is not None:  # memory of the new stream's, that it may be given back behind its work; the old one's, not ahead of the copies
            old = self._step
            with torch.cuda.stream(stream):
                self._step = {k: v.clone() if torch.is_tensor(v) else v for k, v in old.items()}
            for v in old.values():
                if torch.is_tensor(v):
                    v.record_stream(stream)

    # ---- threads (host) ------------------------------------------------------------------------
    def _new_tag(self, request):
        r = self.requests[request]
        for tag in range(TAGS):
            if not (r.used >> tag) & 1:
                r.used |= 1 << tag
                return tag
        raise RuntimeError(f"request {request}: {TAGS} tags are in use; join its threads first")

    def open(self, request) -> Thread:
        """The main thread of an empty request."""
        r = self.requests[request]
        if r.threads:
            raise ValueError(f"request {request} is open")
        tag = self._new_tag(request)
        t = Thread(request, tag, 1 << tag)
        r.threads.append(t)
        return t

    def fork(self, parent: Thread, position=None) -> Thread:
        """A child that sees what `parent` sees now.  `position`: id of its first row (estimated ids may leave gaps); else it counts on."""
        if not parent.alive:
            raise ValueError("forks a living thread")
        self._must_be_settled()
        r = self.requests[parent.request]
        free = TAGS - bin(r.used).count("1")
        if free < 2:
            raise RuntimeError(f"request {parent.request}: {TAGS} tags are in use; join its threads first")
        tag, own = self._new_tag(parent.request), self._new_tag(parent.request)
        child = Thread(parent.request, tag, parent.sees | 1 << tag, parent.position if position is None else position)
        parent.tag, parent.sees = own, parent.sees | 1 << own
        r.threads.append(child)
        return child

    def join(self, thread: Thread, others):
        """`thread` sees from now on what `others` saw; they end.  Their rows stay where they are."""
        r = self.requests[thread.request]
        others = list(others)
        if not thread.alive or len({id(o) for o in others}) != len(others):
            raise ValueError("joins living threads of one request, each once")
        for o in others:
            if o is thread or not o.alive or o.request != thread.request:
                raise ValueError("joins living threads of one request, each once")
        self._must_be_settled()
        for o in others:
            thread.sees |= o.sees
            o.alive = False
            r.threads.remove(o)
        if len(r.threads) == 1:
            # everything written is seen: a prefix, as long as the device says (a step may have been refused), and the tags are free again
            r.used, thread.tag, thread.sees = 1, 0, 1
            self._take_back()
            self._on_stream(lambda: self.prefix_len[thread.request].copy_(self.length[thread.request]))

    def release(self, request):
        """Ends the request's threads and gives its pages back."""
        self._take_back()
        r = self.requests[request]
        for t in r.threads:
            t.alive = False
        self.requests[request] = _Request()
        n = len(self.requests)

        def give_back():
            self.prefix_len[request].zero_()
            keep = self.length.clone()
            keep[request].zero_()
            self.handle.slots(self.length, torch.zeros(n + 1, dtype=torch.int32, device=self.device), 0, None, self.length, self.free_count,
                              self.free_count, keep=keep)
            self._keep_all()
        self._on_stream(give_back)

    def _take_back(self):
        """Drafts that were not accepted, ahead of the next step.  In a call of its own: of a request that slots refuses nothing changes, its rejected drafts
        would stay, and what it keeps would become all of them."""
        def take():
            self.handle.slots(self.length, self._no_rows, 0, None, self.length, self.free_count, self.free_count, keep=self.keep)
            self._keep_all()
        if self.keep is not None:
            self._on_stream(take)

    def _keep_all(self):
        if self.keep is not None:
            self.keep.copy_(self.length)

    def _must_be_settled(self):
        if self._unsettled:
            raise RuntimeError("a verified step's threads do not know their positions: settle() first")

    def _on_stream(self, what):
        with torch.cuda.stream(self._stream):
            what()

    # ---- a step --------------------------------------------------------------------------------
    def begin(self, rows, positions=None):
        """Places of a step's rows: `rows` names the thread of each, requests ascending (a thread may write several).  `positions`: their ids.

        A request that the cache has no room for is refused on the device, which the host does not wait for: the positions of its threads go on as if it
        had been served, until refused() sets them back."""
        self._must_be_settled()
        n = len(rows)
        where = [t.request for t in rows]
        if where != sorted(where) or not all(t.alive for t in rows):
            raise ValueError("rows of living threads, requests ascending")
        count = [0] * len(self.requests)
        ids, after = [], {id(t): t.position for t in rows}
        for i, t in enumerate(rows):
            count[t.request] += 1
            ids.append(after[id(t)] if positions is None else int(positions[i]))
            after[id(t)] = ids[-1] + 1
        offsets = [0]
        for k in count:
            offsets.append(offsets[-1] + k)
        dev = lambda x, t: torch.tensor(x, dtype=t).to(self.device)  # noqa: E731
        signed = [t.sees - (1 << 64) if t.sees >> 63 else t.sees for t in rows]
        times = Counter(id(t) for t in rows)
        self._on_stream(lambda: self._enter(dict(
            n=n, most=max(count), rows=list(rows), threads=set(times), verified=False, offsets=dev(offsets, torch.int32), tag=dev([t.tag for t in rows], torch.uint8), see=dev(signed, torch.int64),
            position=dev(ids, torch.int32), stride=dev([times[id(t)] for t in rows], torch.int32))))
        for t in rows:
            t.position = after[id(t)]

    def _enter(self, step):
        for c in self._captured:
            if c["verified"] and c is not step and not c["threads"].isdisjoint(step["threads"]):
                c["verified"] = False  # (its threads go on elsewhere, and know their positions from there)
        if torch.cuda.is_current_stream_capturing():
            self._captured.append(step)
        if self.keep is not None:
            self.handle.slots(self.length, self._no_rows, 0, None, self.length, self.free_count, self.free_count, keep=self.keep)  # (_take_back)
            step["next"] = torch.add(step["position"], step["stride"], out=step.get("next"))
        self.handle.slots(self.length, step["offsets"], step["n"], self.slot, self.length, self.free_count, self.free_count, row_tag=step["tag"],
                          row_position=step["position"])
        self._keep_all()
        (self.cache or self.handle).plan(self.length, step["offsets"], step["n"], max_request_rows=step["most"], prefix_len=self.prefix_len, slot=self.slot)
        self._step = step
        step["refused"] = None  # (not known)

    def again(self):
        """The step's threads once more, each as many rows further as it has in the step: what a replayed graph does.

        Captured, the step goes on with rows, tags and positions of its own for as long as the session lives.  They are those of the capture: between
        replays its threads neither fork nor join nor write rows by other calls.  What other requests do is free."""
        def go_on():
            if self.keep is not None:  # (verify() has a say in it)
                self._step["position"].copy_(self._step["next"])
            else:
                self._step["position"].add_(self._step["stride"])
            self._enter(self._step)
        self._on_stream(go_on)

    def refused(self):
        """The requests that the last step begun, or gone on with by a call of again(), was refused for (waits for the device).  Their threads' next rows get
        the ids of the refused ones."""
        s = self._step
        if s["refused"] is None:
            with torch.cuda.stream(self._stream):
                slot, ids = self.slot[:s["n"]].tolist(), s["position"].tolist()
                first = {}
                for i, t in enumerate(s["rows"]):
                    first.setdefault(t.request, i)
                s["refused"] = sorted(r for r, i in first.items() if slot[i] < 0)
                for i in reversed(range(s["n"])):  # (of a thread's rows the first one's)
                    t = s["rows"][i]
                    if t.request in s["refused"]:
                        t.position = ids[i]
                        if self.keep is not None:
                            s["next"][i] = s["position"][i]
                        else:
                            s["position"][i] -= s["stride"][i]  # (again() adds it)
        return s["refused"]

    def advanced(self, rows, steps):
        """Tells the host that `steps` calls or replays of again() with these rows have been enqueued."""
        for t in rows:
            t.position += steps

    def layer(self, layer, k_new, v_new, q, out, lse=None):
        """Appends the step's rows of a layer, then attends: row i sees its own row too.  With rope, q and k come as they are, and are turned here."""
        s, cache = self._step, self.cache or self.handle
        with torch.cuda.device(self.device):  # (a launch goes by the current device; the stream is the handle's)
            if self.rows is not None and self.rows_cfg.rope_dims:
                n = s["n"]
                self.rows.rotate(s["position"], q, self._q[:n], k_new, self._k[:n], n_rows=n)
                q, k_new = self._q[:n], self._k[:n]
            cache.append(layer, self.slot, k_new, v_new, n_rows=s["n"])
            cache.attend(layer, q, out, lse=lse, logit_cap=self.logit_cap, slopes=self.slopes, row_see=s["see"],
                         row_position=s["position"] if self.slopes is not None else None)

    def verify(self, token, target, draw, last_draw, draft=None):
        """Holds the step's rows to the target's probabilities: of each request's rows, those of one thread (what is not accepted goes from the request's end, where
        the rows of several threads would lie in turn), the first is its last token and the others drafts.
        token, draw [n]; target, draft [n, vocab]; last_draw [max_requests].  Returns (accepted, next token) of every request, on the device, until the next call.

        The next begin() or again() takes back what was not accepted.  again() goes on behind the accepted rows without the host; begin(), fork() and join()
        want settle() first, also behind replays of a captured step that ends with verify()."""
        s = self._step
        if self.keep is None or s is None:
            raise RuntimeError("verify() wants a session with vocab and a step that has begun")
        owner = {}
        for t in s["rows"]:
            if owner.setdefault(t.request, t) is not t:
                raise ValueError(f"request {t.request}: rows of several threads are no drafts")
        with torch.cuda.device(self.device):
            self.rows.verify(s["offsets"], token, target, draw, last_draw, self.accepted, self.next_token, draft=draft, length=self.length, keep=self.keep,
                             row_position=s["position"], position_out=s["next"], slot=self.slot, n_sequences=len(self.requests), n_rows=s["n"])
        s["verified"] = self._unsettled = True
        return self.accepted, self.next_token

    def settle(self):
        """Waits for the device, after verify() or replays that end with it, and tells the threads of such steps their positions.  Returns the requests'
        accepted drafts."""
        if self.keep is None:
            raise RuntimeError("settle() wants a session with vocab")
        with torch.cuda.stream(self._stream):
            # (the last step, which may be a copy of a captured one, ahead of those, which replays have moved on)
            for s in [s for s in (self._step, *self._captured) if s is not None and s["verified"]]:
                ids = s["next"].tolist()
                for i in reversed(range(s["n"])):  # (of a thread's rows the first one's)
                    s["rows"][i].position = ids[i]
            self._unsettled = False
            return self.accepted.tolist()


def main():
    """A prompt, three threads, and thirty-two of their steps as replays of one captured step; then the join."""
    torch.manual_seed(0)
    layers, hq, hkv, d, n = 4, 32, 8, 128, 3
    s = Session(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, softmax_scale=d ** -0.5, n_layers=layers, max_rows=512, n_phys_pages=256, pages_per_request=128)
    randn = lambda *shape: torch.randn(*shape, device="cuda", dtype=torch.bfloat16)  # noqa: E731

    def forward(rows):
        q, k, v = randn(layers, rows, hq, d), randn(layers, rows, hkv, d), randn(layers, rows, hkv, d)
        out = torch.empty_like(q)
        for l in range(layers):
            s.layer(l, k[l], v[l], q[l], out[l])
        return out, (q, k, v)

    root = s.open(0)
    s.begin([root] * 300)
    forward(300)
    threads = [s.fork(root) for _ in range(n)]
    s.begin(threads)
    forward(n)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        s.bind(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            s.again()
            out, _keep = forward(n)
        for _ in range(32):
            graph.replay()
    stream.synchronize()
    s.advanced(threads, 32)
    s.bind(torch.cuda.current_stream())
    s.join(root, threads)
    s.begin([root])
    out, _keep = forward(1)
    torch.cuda.synchronize()
    print("tokens", int(s.length[0]), "pages left", int(s.free_count), "output", float(out.float().norm()))


if __name__ == "__main__":
    main()
