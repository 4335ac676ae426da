"""Sessions that draw under top-k, top-p and min-p, in every kernel family: a step's rows are masked as the oracle masks the logits of the same step without
filters, and its acceptance is the oracle's on them; top-k 1 is greedy decoding; without filters all is as before."""
import numpy as np
import pytest

import workload as W
from oracle import filtered_sampling as OF
from oracle import sampled_acceptance as OA
from test_gpu_sampled_decoding import MODELS, randoms, rig_of

pytestmark = pytest.mark.gpu


def settings(B):
    import torch
    dev = lambda v, t: torch.tensor((v * B)[:B], dtype=t, device="cuda")
    return dev([0, 7, 40, 0, 3], torch.int32), dev([0.7, 1.0, 0.9, 0.95, 0.5], torch.float32), dev([0.0, 0.0, 0.02, 0.1, 0.0], torch.float32)


@pytest.mark.parametrize("name", list(MODELS))
def test_a_step(name):
    import torch
    rig = rig_of(name)
    T, cfg, B, k = rig.T, rig.cfg, rig.batch, rig.cfg.k
    u = randoms(B, 12)
    temperature = torch.tensor([0.9, 0.5, 0.0, 1.3][:B] * B, device="cuda")[:B].contiguous()
    filters = settings(B)
    T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, 12)
    drafts = torch.zeros((B, k), dtype=torch.int32, device="cuda")
    accept, emitted, logprob = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, k + 1), dtype=torch.int32, device="cuda"), torch.zeros((B, k + 1), device="cuda")
    scratch = torch.zeros(T.tasc_sampled_scratch_bytes(rig.model, B, k), dtype=torch.uint8, device="cuda")

    def step():
        print(name, flush=True)
        T.tasc_session_rewind(rig.session)
        T.tasc_draft(rig.ng, rig.session, rig.params(), drafts)
        T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, u, temperature, accept, emitted, logprob, scratch)
        z = scratch[:B * (k + 1) * cfg.vocab * 4].view(torch.float32).view(B, k + 1, cfg.vocab).cpu().numpy()
        return z, accept.tolist(), emitted.tolist(), logprob.cpu().numpy().copy()

    raw = step()
    T.tasc_session_filter(rig.session, *filters)
    tk, tp, mp = (f.tolist() for f in filters)
    for _ in range(3):                                      # launched, recorded, replayed
        z, m, tokens, logp = step()
        for b in range(B):
            want = np.stack([OF.masked(raw[0][b, i], float(temperature[b]), tk[b], np.float32(tp[b]), np.float32(mp[b]))[0] for i in range(k + 1)])
            assert np.array_equal(z[b], want)
            n, out, lp = OA.accept(want, drafts[b].cpu().numpy(), None, float(temperature[b]), u[b, :k + 1].cpu().numpy())
            assert m[b] == n and tokens[b] == out + [-1] * (k - n)
            assert np.abs(logp[b][:n + 1] - lp).max() <= 2.0 ** -24 * np.abs(lp).max() + 1e-12
    T.tasc_session_filter(rig.session)
    again = step()
    assert np.array_equal(again[0], raw[0]) and again[1:3] == raw[1:3]


@pytest.mark.parametrize("cache", ["model", "kv4"])
@pytest.mark.parametrize("name", list(MODELS))
def test_top_k_1_is_greedy(name, cache):
    import torch
    if cache == "kv4" and name == "f32":
        pytest.skip("4-bit caches are of bf16 models")
    rig = rig_of(name)
    T, cfg, B = rig.T, rig.cfg, rig.batch
    if cache == "kv4":
        rig.session = T.tasc_session_create_kv4(rig.model, B, rig.max_len, rig.max_rows, B * (rig.max_len // 16 + 1))
    greedy = rig.generate(k=0)[0]
    T.tasc_session_filter(rig.session, top_k=torch.ones(B, dtype=torch.int32, device="cuda"))
    for k in (0, cfg.k):
        out = torch.zeros((B, cfg.gen_len), dtype=torch.int32, device="cuda")
        T.tasc_generate_sampled(rig.model, rig.ng if k else None, rig.session, rig.prompts, rig.prompt_off, cfg.gen_len, rig.params(k), randoms(B, cfg.gen_len), out,
                                torch.full((B,), 1.5, device="cuda"))
        assert np.array_equal(out.cpu().numpy(), greedy)


def test_recorded_steps_are_the_plain_ones():
    """Steps with filters and without in turn, recorded and replayed, on one session"""
    import torch
    rig = rig_of("tiled")
    T, cfg, B = rig.T, rig.cfg, rig.batch
    filters = settings(B)
    outs = []
    try:
        for graph in (0, 1):
            T.tasc_config_set(T.TASC_CFG_STEP_GRAPH, graph)
            for on in (True, False, True):
                T.tasc_session_filter(rig.session, *(filters if on else ()))
                out = torch.zeros((B, cfg.gen_len), dtype=torch.int32, device="cuda")
                T.tasc_generate_sampled(rig.model, rig.ng, rig.session, rig.prompts, rig.prompt_off, cfg.gen_len, rig.params(), randoms(B, cfg.gen_len, 3), out)
                outs.append(out.cpu().numpy())
    finally:
        T.tasc_config_set(T.TASC_CFG_STEP_GRAPH, 1)
    for i in range(3):
        assert np.array_equal(outs[i], outs[3 + i])
    assert np.array_equal(outs[0], outs[2]) and not np.array_equal(outs[0], outs[1])


def test_a_workspace_that_is_too_small():
    import torch
    rig = rig_of("tiled")
    T, B, k = rig.T, rig.batch, rig.cfg.k
    need = T.tasc_sample_workspace_bytes(B * (k + 1), rig.cfg.vocab)
    assert need > 0
    T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, 4)
    T.tasc_session_filter(rig.session, top_k=torch.ones(B, dtype=torch.int32, device="cuda"), workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
    drafts = torch.zeros((B, k), dtype=torch.int32, device="cuda")
    with pytest.raises(T.TascError):
        T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, randoms(B, 4))
    T.tasc_session_filter(rig.session)
    T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, randoms(B, 4))


def test_filters_that_are_replaced_while_a_step_is_under_way():
    """The old filters' memory is free for others only when the steps that were enqueued with them, on whatever stream, have ended"""
    import torch
    rig = rig_of("tiled")
    T, B, k = rig.T, rig.batch, rig.cfg.k
    u = randoms(B, 8)
    drafts = torch.zeros((B, k), dtype=torch.int32, device="cuda")
    accept, emitted = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, k + 1), dtype=torch.int32, device="cuda")
    scratch = torch.zeros(T.tasc_sampled_scratch_bytes(rig.model, B, k), dtype=torch.uint8, device="cuda")
    a, b = torch.zeros(1 << 28, dtype=torch.uint8, device="cuda"), torch.zeros(1 << 28, dtype=torch.uint8, device="cuda")
    T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, 12)
    side = torch.cuda.Stream()
    outs = []
    for busy in (False, True):
        T.tasc_session_rewind(rig.session)
        T.tasc_session_filter(rig.session, top_k=torch.full((B,), 2, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        for _ in range(50 if busy else 0):                  # (6 ms)
            T.tasc_calibration_copy(a, b, stream=side.cuda_stream)
        T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, u, None, accept, emitted, None, scratch, stream=side.cuda_stream)
        if busy:
            T.tasc_session_filter(rig.session)
            other = [torch.full((B,), 1000, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        z = scratch[:B * (k + 1) * rig.cfg.vocab * 4].view(torch.float32).view(B, k + 1, rig.cfg.vocab)
        assert ((z > float("-inf")).sum(2) == 2).all()
        outs.append((accept.tolist(), emitted.tolist()))
    assert outs[0] == outs[1]


def test_filters_that_overlap_what_a_step_writes():
    """Refused before anything of the step is enqueued"""
    import torch
    rig = rig_of("tiled")
    T, B, k = rig.T, rig.batch, rig.cfg.k
    u = randoms(B, 4)
    drafts = torch.zeros((B, k), dtype=torch.int32, device="cuda")
    ws = torch.zeros(T.tasc_sample_workspace_bytes(B * (k + 1), rig.cfg.vocab), dtype=torch.uint8, device="cuda")
    scratch = torch.zeros(T.tasc_sampled_scratch_bytes(rig.model, B, k) + ws.numel(), dtype=torch.uint8, device="cuda")       # (room for both)
    ones = lambda at: at[256:256 + 4 * B].view(torch.int32).fill_(1)
    accept, emitted = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, k + 1), dtype=torch.int32, device="cuda")
    step = lambda: T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, u, None, accept, emitted, None, scratch)
    T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, 4)
    T.tasc_session_rewind(rig.session)
    step()
    want = accept.tolist(), emitted.tolist()
    T.tasc_session_rewind(rig.session)
    for top_k, workspace in ((ones(ws), ws), (ones(scratch), ws), (ones(torch.zeros(1024, dtype=torch.uint8, device="cuda")), scratch)):
        T.tasc_session_filter(rig.session, top_k=top_k, workspace=workspace)
        with pytest.raises(T.TascError, match="overlap"):
            step()
    T.tasc_session_filter(rig.session)
    step()
    assert (accept.tolist(), emitted.tolist()) == want
