"""Calls on a caller's stream while the current stream still works on memory that
the program let go of: outputs and workspaces must not lie there."""
import pytest
import torch

import padoc_synth as syn
import paper_2608_06146_amd as pa
from _rotary import Setup, normal, positions

pytestmark = pytest.mark.gpu


def leave(shapes, dtype):
    """Tensors that the current stream writes some milliseconds from now, let go
    of; returns their addresses."""
    ts = [torch.empty(s, dtype=t, device="cuda") for s, t in zip(shapes, dtype)]
    torch.cuda._sleep(2_000_000)
    for t in ts:
        t.fill_(7)
    return {t.data_ptr() for t in ts}


def rotary_calls():
    st, n, hq, hkv, d = Setup(64, "bf16"), 3000, 8, 2, 64
    q, k, v = normal((n, hq, d), 1, "bf16"), normal((n, hkv, d), 2, "bf16"), normal((n, hkv, d), 3, "bf16")
    w, pos = normal((d,), 4, "bf16"), positions(3, n, 5)
    nb = -(-n // 16)
    t = torch.arange(n, dtype=torch.int32)
    slots = torch.stack([t // 16, t % 16], 1).cuda()
    kc, vc = torch.zeros((nb, hkv, d // 8, 16, 8), dtype=q.dtype, device="cuda"), torch.zeros((nb, hkv, d, 16), dtype=q.dtype, device="cuda")
    return {"fwd": lambda s: pa.rotary_fwd(q, k, pos, st.handle, w, w, stream=s),
            "bwd": lambda s: pa.rotary_bwd(q, k, pos, st.handle, q, k, w, w, stream=s),
            "append": lambda s: (pa.rotary_append(q, k, v, pos, slots, kc, vc, st.handle, w, w, stream=s), kc, vc)}


def on_a_busy_device(call):
    """``call(side)`` beside queued work on memory of its outputs' sizes gives
    what ``call(None)`` gives."""
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    shapes, types = [t.shape for t in want], [t.dtype for t in want]
    torch.cuda.synchronize()
    for i in range(3):
        print("[case] run", i, flush=True)
        left = leave(shapes, types)
        got = call(side)
        assert not left & {t.data_ptr() for t in got}
        side.synchronize()
        torch.cuda.synchronize()  # the queued writes too
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got


@pytest.mark.parametrize("what", ["fwd", "bwd", "append"])
def test_rotary_calls(what):
    on_a_busy_device(rotary_calls()[what])


@pytest.mark.parametrize("form", ["plain", "rotary"])
def test_a_growing_session(form):
    """Steps that outgrow the session's workspace on a stream of the caller's;
    between them the current stream allocates and writes as much memory.  The
    results are those of a twin that runs alone."""
    hq, hkv, d, nb = 8, 2, 64, 700
    st, w = Setup(d, "bf16"), normal((d,), 1, "bf16")

    def session():
        kc, vc = torch.zeros((nb, hkv, d // 8, 16, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((nb, hkv, d, 16), dtype=torch.bfloat16, device="cuda")
        return pa.DecodeSession(hq, hkv, d, nb, "bf16", kc, vc, torch.zeros(4096, dtype=torch.int32, device="cuda"))

    steps = [(1, 40), (3, 5), (20, 9), (64, 3), (64, 30)]  # streams, tokens of each
    rows = [(normal((s * t, hq, d), i, "bf16"), normal((s * t, hkv, d), i + 20, "bf16"), positions(3, s * t, i)) for i, (s, t) in enumerate(steps)]

    def run(stream):
        s, out, sizes = session(), [], []
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        for (n, t), (q, k, pos) in zip(steps, rows):
            while s.n_open < n:
                s.open()
            s.prepare([t] * n, [t] * n)
            print("[case]", form, n, t, s.workspace_bytes, flush=True)
            sizes.append(s.workspace_bytes)
            out.append(s.launch_rotary(q, k, k, pos, st.handle, w, w, stream=stream) if form == "rotary" else s.launch(q, k, k, stream=stream))
            if stream is not None:
                for z in sizes:
                    torch.full((z + z // 4 + 256,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        assert max(sizes) > 2 * sizes[0]
        return [t for o in out for t in o] + [s.k_cache, s.v_cache]

    want = run(None)
    got = run(torch.cuda.Stream())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def attention_calls():
    hq, hkv, d = 8, 2, 64
    pages = [syn.Page(150, 150, 40, 40, (syn.Branch(7, 90, 90), syn.Branch(25, 45, 45)))] * 3
    n = syn.count_tokens(pages)
    plan = pa.TreePlan(pa.segments_from_pages(pages, 0), hq, hkv, d, "bf16", 0, num_kv_rows=n, num_q_rows=n)
    q, k, v, g = normal((n, hq, d), 1, "bf16"), normal((n, hkv, d), 2, "bf16"), normal((n, hkv, d), 3, "bf16"), normal((n, hq, d), 4, "bf16")
    o, lse = pa.tree_attn_fwd(q, k, v, plan)
    lens = [33, 70, 5]
    segs = pa.segments_layout([(-1, 0, t, 1) for t in lens], 16)
    nb = sum(-(-t // 16) for t in lens)
    decode = pa.TreePlan(segs, hq, hkv, d, "bf16", 16, num_kv_rows=nb, block_table_len=nb)
    rows = normal((nb, hkv, 16, d), 5, "bf16")
    kc, vc = pa.cache_from_rows(rows, rows)
    table = torch.arange(nb, dtype=torch.int32, device="cuda")
    return {"forward": lambda s: pa.tree_attn_fwd(q, k, v, plan, stream=s),
            "backward": lambda s: pa.tree_attn_bwd(q, k, v, o, lse, g, plan, stream=s),
            "decode": lambda s: pa.branch_decode(q[:3], kc, vc, table, decode, stream=s),
            "cache": lambda s: pa.cache_from_rows(rows, rows, stream=s)}


@pytest.mark.parametrize("what", ["forward", "backward", "decode", "cache"])
def test_attention_calls(what):
    on_a_busy_device(attention_calls()[what])


def test_captured_on_a_forked_stream():
    """Calls on a stream that a capture forked to, replayed with the program's
    own work between."""
    st, n, d = Setup(64, "bf16"), 700, 64
    q, w, pos = normal((n, 8, d), 1, "bf16"), normal((d,), 2, "bf16"), positions(3, n, 3)
    run = lambda s: [*pa.rotary_fwd(q, None, pos, st.handle, w, stream=s)[:1], *pa.rotary_bwd(q, None, pos, st.handle, q, None, w, stream=s)[::2]]  # noqa: E731
    run(None)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = run(side)
        torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        q.copy_(normal((n, 8, d), 10 + i, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, run(None))), i


def test_given_outputs_on_a_stream():
    """Attention with every buffer the caller's."""
    hq, hkv, d, n = 8, 2, 64, 150
    plan = pa.TreePlan(pa.segments_layout([(-1, 0, n, n)], 0), hq, hkv, d, "bf16", 0, num_kv_rows=n, num_q_rows=n)
    q, k = normal((n, hq, d), 1, "bf16"), normal((n, hkv, d), 2, "bf16")
    o, lse = pa.tree_attn_fwd(q, k, k, plan)
    grads = pa.tree_attn_bwd(q, k, k, o, lse, q, plan)
    out, l2, g2 = torch.zeros_like(o), torch.zeros_like(lse), [torch.zeros_like(t) for t in grads]
    ws, bws = plan.workspace("cuda"), plan.backward_workspace("cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pa.tree_attn_fwd(q, k, k, plan, out, l2, ws, stream=side)
    pa.tree_attn_bwd(q, k, k, out, l2, q, plan, *g2, bws, stream=side)
    side.synchronize()
    assert torch.equal(o, out) and torch.equal(lse, l2) and all(torch.equal(a, b) for a, b in zip(grads, g2))
