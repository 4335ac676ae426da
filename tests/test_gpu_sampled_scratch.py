"""The scratch of sampled steps: whose memory it is, and what is refused."""
import numpy as np
import pytest

from test_gpu_sampled_decoding import randoms, rig_of

pytestmark = pytest.mark.gpu


def owner(t):
    """The stream whose memory a tensor lies in."""
    import torch
    at = t.data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


def test_scratch_of_the_stream_that_uses_it():
    """Memory that the current stream freed may still be written by what is enqueued there: a step on another stream does not get it.  What it
    computes is what the current stream's step computes."""
    import torch
    rig = rig_of("tiled")
    T, B, k = rig.T, rig.batch, rig.cfg.k
    u, drafts = randoms(B, 6), torch.zeros((B, k), dtype=torch.int32, device="cuda")
    emitted = torch.zeros((B, k + 1), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    got = []
    for st in (None, side.cuda_stream, None, side.cuda_stream):
        torch.empty(T.tasc_sampled_scratch_bytes(rig.model, B, k), dtype=torch.uint8, device="cuda")     # freed at once
        T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, 6)
        T.tasc_session_rewind(rig.session)
        torch.cuda.synchronize()
        for _ in range(3):                                    # (the third one is a recorded step)
            T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, u, emitted=emitted, stream=st)
        torch.cuda.synchronize()
        got.append([T.tasc_session_get_tokens(rig.session, b).tolist() for b in range(B)])
    assert all(g == got[0] for g in got)
    assert {owner(t) for t in rig.session._scratch.values()} == {torch.cuda.current_stream().cuda_stream, side.cuda_stream}
    out = torch.zeros((B, 6), dtype=torch.int32, device="cuda")
    runs = []
    for st in (None, side.cuda_stream):
        torch.cuda.synchronize()
        T.tasc_generate_sampled(rig.model, rig.ng, rig.session, rig.prompts, rig.prompt_off, 6, rig.params(), u, out, stream=st)
        torch.cuda.synchronize()
        runs.append(out.cpu().numpy().copy())
    assert (runs[0] == runs[1]).all()
    assert all(owner(t) == st for (_, st), t in rig.session._scratch.items())


def test_scratch_that_is_refused():
    import torch
    rig = rig_of("f32")
    T, B = rig.T, rig.batch
    u, drafts = randoms(B, 4), torch.zeros((B, 4), dtype=torch.int32, device="cuda")
    T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, 5)
    n = T.tasc_sampled_scratch_bytes(rig.model, B, 4)
    wide = torch.zeros((n, 2), dtype=torch.uint8, device="cuda")
    before = [T.tasc_session_get_tokens(rig.session, b).tolist() for b in range(B)]
    for bad in (torch.zeros(n, dtype=torch.uint8), wide[:, 0], np.zeros(n, dtype=np.uint8), wide.data_ptr()):
        with pytest.raises(T.TascError):
            T.tasc_verify_step_sampled(rig.model, rig.session, drafts, 4, u, scratch=bad)
        with pytest.raises(T.TascError):
            T.tasc_generate_sampled(rig.model, rig.ng, rig.session, rig.prompts, rig.prompt_off, 5, rig.params(4), u,
                                    torch.zeros((B, 5), dtype=torch.int32, device="cuda"), scratch=bad)
    assert [T.tasc_session_get_tokens(rig.session, b).tolist() for b in range(B)] == before


def test_recorded_by_the_caller():
    """Steps that a program records itself, in two graphs of which the first is dropped; replays with eager steps in between."""
    import gc
    import torch
    rig = rig_of("tiled")
    T, B, k = rig.T, rig.batch, rig.cfg.k
    u, drafts = randoms(B, 12), torch.zeros((B, k), dtype=torch.int32, device="cuda")

    def begin():
        T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, 12)
        T.tasc_session_rewind(rig.session)
        torch.cuda.synchronize()

    def tokens():
        torch.cuda.synchronize()
        return [T.tasc_session_get_tokens(rig.session, b).tolist() for b in range(B)]

    def step():
        T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, u)

    begin()
    want = []
    for _ in range(6):
        step()
        want.append(tokens())
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    for g in (first, second):
        with torch.cuda.graph(g):
            step()
    del first, g
    gc.collect()
    torch.cuda.empty_cache()
    for again in range(2):
        begin()
        for at in range(6):
            noise = torch.full((1 << 26,), float("nan"), device="cuda")      # whoever's memory is not its own sees these
            if at % 3 == 2:
                step()
            else:
                second.replay()
            assert tokens() == want[at], (again, at)
            del noise
