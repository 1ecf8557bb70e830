"""Whose memory a call on a caller's stream uses: what it allocates has to come
from that stream's pool (a block of the current stream's may still be in use by
work queued there), and what it returns or a session keeps has to stay while any
stream uses it.  On the CPU, with stand-ins for the allocator and the launches."""
import pytest
import torch

import paper_2608_06146_amd as pa
from _streams import Gpu, addresses


def words_of(*args):
    for a in args:
        if isinstance(a, bytes):
            yield from addresses(a)
        elif a is not None:
            yield int(getattr(a, "value", a) or 0)


def calls_of_rows(gpu, rot, side):
    """Every rotary call with outputs of its own on stream ``side``."""
    t = lambda *shape, dtype=torch.bfloat16: gpu.tensor(torch.zeros(shape, dtype=dtype))  # noqa: E731
    q, k, v, w, pos = t(6, 4, 64), t(6, 2, 64), t(6, 2, 64), t(64), t(3, 6, dtype=torch.int32)
    slots, kc, vc = t(6, 2, dtype=torch.int32), t(3, 2, 8, 16, 8), t(3, 2, 64, 16)
    return {"fwd": lambda: pa.rotary_fwd(q, k, pos, rot, w, w, stream=side),
            "bwd": lambda: pa.rotary_bwd(q, k, pos, rot, q, k, w, w, stream=side),
            "append": lambda: pa.rotary_append(q, k, v, pos, slots, kc, vc, rot, w, w, stream=side)}


@pytest.mark.parametrize("what", ["fwd", "bwd", "append"])
def test_rotary_calls_allocate_on_the_callers_stream(monkeypatch, what):
    seen = []
    call = lambda *a: seen.append(a) or 0  # noqa: E731
    gpu = Gpu(monkeypatch, {f"padoc_rotary_{w}": call for w in ("fwd", "bwd", "append")})
    rot = pa.Rotary(64, "bf16", sections=(8, 12, 12))
    run = calls_of_rows(gpu, rot, gpu.side)[what]
    given = len(gpu.made)
    out = run()
    assert gpu.current is gpu.first
    made = gpu.made[given:]
    assert made and all(t.allocated is gpu.side for t in made)
    assert len(seen) == 1 and seen[0][-1] == gpu.side.cuda_stream
    words = set(words_of(*seen[0][1:-1]))
    assert all(t.data_ptr() in words for t in made)
    # what the caller gets is read on the stream that is current there
    for t in out if isinstance(out, tuple) else (out,):
        assert any(t is m for m in made) and gpu.first in t.recorded


def test_given_outputs_stay_the_callers(monkeypatch):
    gpu = Gpu(monkeypatch, {"padoc_rotary_fwd": lambda *a: 0, "padoc_cache_copy_blocks": lambda *a: 0})
    rot = pa.Rotary(64, "bf16")
    q, o, pos = (gpu.tensor(torch.zeros(s, dtype=d)) for s, d in (((5, 4, 64), torch.bfloat16), ((5, 4, 64), torch.bfloat16), ((5,), torch.int32)))
    kc, vc = (gpu.tensor(torch.zeros(s, dtype=torch.bfloat16)) for s in ((3, 2, 8, 16, 8), (3, 2, 64, 16)))
    pairs = gpu.tensor(torch.zeros((1, 2), dtype=torch.int32))
    given = len(gpu.made)
    assert pa.rotary_fwd(q, None, pos, rot, q_out=o, stream=gpu.side)[0] is o
    assert pa.cache_copy_blocks(kc, vc, pairs, stream=gpu.side) == (kc, vc)
    assert len(gpu.made) == given and not any(t.recorded for t in gpu.made)


class Serving:
    """A session whose launches note the memory they were given and end at once."""

    def __init__(self, monkeypatch):
        self.seen = []
        names = ("padoc_session_launch", "padoc_session_launch_rotary")
        self.gpu = gpu = Gpu(monkeypatch, {n: self.launched for n in names})
        t = lambda *shape, dtype=torch.bfloat16: gpu.tensor(torch.zeros(shape, dtype=dtype))  # noqa: E731
        self.t = t
        self.caches = t(40, 2, 8, 16, 8), t(40, 2, 64, 16), t(256, dtype=torch.int32)
        self.s = pa.DecodeSession(4, 2, 64, 40, "bf16", *self.caches)
        self.rot = pa.Rotary(64, "bf16")

    def launched(self, *a):
        self.seen.append(a)
        self.s.commit()
        return 0

    def step(self, form, n, stream):
        self.s.prepare([n] * self.s.n_open, [n] * self.s.n_open)
        n *= self.s.n_open
        q, k, v = self.t(n, 4, 64), self.t(n, 2, 64), self.t(n, 2, 64)
        given = len(self.gpu.made)
        if form == "rotary":
            out = self.s.launch_rotary(q, k, v, self.t(n, dtype=torch.int32), self.rot, stream=stream)
            given += 1
        else:
            out = self.s.launch(q, k, v, stream=stream)
        return out, self.gpu.made[given:]


def test_a_sessions_rotary_launch_allocates_on_the_callers_stream(monkeypatch):
    sv = Serving(monkeypatch)
    sv.s.open()
    out, made = sv.step("rotary", 5, sv.gpu.side)
    assert len(made) == 4 and all(t.allocated is sv.gpu.side for t in made)  # out, lse, rotated queries, workspace
    assert all(sv.gpu.first in t.recorded for t in out)


@pytest.mark.parametrize("form", ["plain", "rotary"])
def test_a_session_keeps_its_memory_for_the_steps_queued(monkeypatch, form):
    """Steps on two streams, growing: whatever the session holds was allocated
    on, or recorded for, every stream that a step ran on."""
    sv = Serving(monkeypatch)
    for _ in range(4):
        sv.s.open()
    held = []
    for n, stream in ((1, None), (1, sv.gpu.side), (60, sv.gpu.side), (1, None), (80, None)):
        sv.step(form, n, stream)
        s = stream or sv.gpu.first
        address = sv.seen[-1][5 if form == "rotary" else 6]
        workspace = sv.gpu.holder(getattr(address, "value", address))
        if not any(workspace is t for t in held):
            held.append(workspace)
        for t in (workspace, *sv.caches):
            assert t.allocated is s or s in t.recorded
    assert len(held) >= 2  # outgrown and replaced


def test_caches_that_a_session_is_moved_from(monkeypatch):
    sv = Serving(monkeypatch)
    sv.s.open()
    sv.step("rotary", 5, sv.gpu.side)
    new = sv.t(50, 2, 8, 16, 8), sv.t(50, 2, 64, 16)
    sv.s.resize(50, *new)
    sv.step("rotary", 5, sv.gpu.side)
    assert all(sv.gpu.side in t.recorded for t in (*sv.caches, *new))


def test_a_plain_launch_allocates_on_the_callers_stream(monkeypatch):
    sv = Serving(monkeypatch)
    sv.s.open()
    out, made = sv.step("plain", 5, sv.gpu.side)
    assert len(made) == 3 and all(t.allocated is sv.gpu.side for t in made)  # out, lse, workspace
    assert all(sv.gpu.first in t.recorded for t in out)


ATTENTION = ("padoc_tree_attn_fwd", "padoc_tree_attn_bwd", "padoc_branch_decode", "padoc_cache_from_rows")


@pytest.mark.parametrize("what", ATTENTION)
def test_attention_calls_allocate_on_the_callers_stream(monkeypatch, what):
    seen = []
    gpu = Gpu(monkeypatch, {n: lambda *a: seen.append(a) or 0 for n in ATTENTION})
    t = lambda *shape, dtype=torch.bfloat16: gpu.tensor(torch.zeros(shape, dtype=dtype))  # noqa: E731
    paged = what == "padoc_branch_decode"
    segs = pa.segments_layout([(-1, 0, 20, 4)], 16 if paged else 0)
    plan = pa.TreePlan(segs, 4, 2, 64, "bf16", 16 if paged else 0, num_kv_rows=2 if paged else 20,
                       block_table_len=2 if paged else None)
    n = plan.num_q_rows
    q, lse, k, kc, vc, table = t(n, 4, 64), t(n, 4, dtype=torch.float32), t(20, 2, 64), t(2, 2, 8, 16, 8), t(2, 2, 64, 16), t(2, dtype=torch.int32)
    rows = t(2, 2, 16, 64)
    given = len(gpu.made)
    out = {"padoc_tree_attn_fwd": lambda s: pa.tree_attn_fwd(q, k, k, plan, stream=s),
           "padoc_tree_attn_bwd": lambda s: pa.tree_attn_bwd(q, k, k, q, lse, q, plan, stream=s),
           "padoc_branch_decode": lambda s: pa.branch_decode(q, kc, vc, table, plan, stream=s),
           "padoc_cache_from_rows": lambda s: pa.cache_from_rows(rows, rows, stream=s)}[what]
    got = out(gpu.side)
    made = gpu.made[given:]
    assert made and all(m.allocated is gpu.side for m in made) and seen[0][-1].value == gpu.side.cuda_stream
    assert all(gpu.first in m.recorded for m in got)
    if what != "padoc_cache_from_rows":  # the plan's own workspace, used on another stream next
        out(None)
        assert sum(m.dtype == torch.uint8 for m in gpu.made) == 1
        assert all(gpu.first in m.recorded for m in gpu.made if m.dtype == torch.uint8)
