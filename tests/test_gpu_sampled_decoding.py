"""Sampled decoding in every kernel family: a step's acceptance is the oracle's on the logits that the step left in its scratch, with the
random pair of each generated token; at temperature 0 the loop is the greedy one."""
import numpy as np
import pytest

import workload as W
from oracle import sampled_acceptance as OA

pytestmark = pytest.mark.gpu

MODELS = {
    "f32": dict(batch=3),                                                                    # the type-generic kernels
    "tiled": dict(dtype="bf16", n_layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ffn=448, vocab=5000, batch=28, n_docs=1500, n_max=4),
    "persistent": dict(dtype="bf16", n_layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ffn=448, vocab=5000, batch=2, k=4, n_docs=1500),
}


def rig_of(name, **kw):
    from gpu_util import Rig
    cfg = W.get_config("cfg1").scaled(**dict(dict(MODELS[name], prompt_len=40, gen_len=30, bias_alpha=1.0), **kw))
    return Rig(cfg, max_rows=8 if name == "persistent" else 16)


def randoms(B, n, seed=0):
    import torch
    return torch.tensor(np.random.default_rng(seed).random((B, n, 2)).astype(np.float32), device="cuda")


@pytest.mark.parametrize("alpha", [1.0, 8.0])           # flat rows; rows that follow the corpus, whose drafts are accepted
@pytest.mark.parametrize("name", list(MODELS))
def test_steps_against_the_oracle(name, alpha):
    import torch
    rig = rig_of(name, bias_alpha=alpha)
    T, cfg, B, k = rig.T, rig.cfg, rig.batch, rig.cfg.k
    G = 12
    u = randoms(B, G)
    temperature = torch.tensor([0.0, 0.5, 0.9, 1.3][:B] * B, device="cuda")[:B].contiguous()
    T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, G)
    T.tasc_session_rewind(rig.session)
    drafts = torch.zeros((B, k), dtype=torch.int32, device="cuda")
    accept, emitted = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, k + 1), dtype=torch.int32, device="cuda")
    logprob = torch.zeros((B, k + 1), device="cuda")
    scratch = torch.zeros(T.tasc_sampled_scratch_bytes(rig.model, B, k), dtype=torch.uint8, device="cuda")
    held = [rig.prompts[rig.prompt_off[b]:rig.prompt_off[b + 1]].tolist() for b in range(B)]
    n_prompt, lengths = len(held[0]), set()
    for step in range(7):
        print(f"{name} step {step}", flush=True)
        T.tasc_draft(rig.ng, rig.session, rig.params(), drafts)
        T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, u, temperature, accept, emitted, logprob, scratch)
        z = scratch[:B * (k + 1) * cfg.vocab * 4].view(torch.float32).view(B, k + 1, cfg.vocab).cpu().numpy()
        got, d = emitted.cpu().numpy(), drafts.cpu().numpy()
        for b in range(B):
            done = len(held[b]) - n_prompt
            if done >= G:
                assert accept[b] == 0 and (got[b] == -1).all() and (logprob[b] == 0).all()
                continue
            pairs = u[b].cpu().numpy()[np.minimum(done + np.arange(k + 1), G - 1)]
            m, tokens, logp = OA.accept(z[b], d[b], None, float(temperature[b]), pairs)
            assert accept[b] == m and got[b].tolist() == tokens + [-1] * (k - m)
            assert np.abs(logprob[b].cpu().numpy()[:m + 1] - logp).max() <= 2.0 ** -24 * np.abs(logp).max() + 1e-12
            held[b] += tokens
            lengths.add(m)
            assert T.tasc_session_get_tokens(rig.session, b).tolist() == held[b]
    assert alpha < 8 or max(lengths) > 0, "no draft was accepted: the test compares little"


@pytest.mark.parametrize("name", list(MODELS))
def test_loop(name):
    """Temperature 0: the tokens of greedy decoding.  Otherwise: the same tokens from recorded steps and plain launches, whatever ran before
    on the session, and those of the steps one by one; statistics that add up."""
    import torch
    rig = rig_of(name)
    T, cfg, B = rig.T, rig.cfg, rig.batch
    out = torch.zeros((B, cfg.gen_len), dtype=torch.int32, device="cuda")
    greedy = rig.generate(k=0)[0]

    def sampled(k, temperature, u=randoms(B, cfg.gen_len)):
        st = T.tasc_generate_sampled(rig.model, rig.ng if k else None, rig.session, rig.prompts, rig.prompt_off, cfg.gen_len, rig.params(k), u, out,
                                     None if temperature is None else torch.full((B,), temperature, device="cuda"))
        assert st.emitted == B * cfg.gen_len and st.accepted == sum(i * n for i, n in enumerate(st.accept_hist)) and st.steps >= cfg.gen_len / (k + 1)
        return out.cpu().numpy().copy()

    for k in (0, cfg.k):
        assert (sampled(k, 0.0) == greedy).all()
    runs = []
    try:
        for graph in (1, 0, 1):
            T.tasc_config_set(T.TASC_CFG_STEP_GRAPH, graph)
            runs.append([sampled(cfg.k, t) for t in (0.8, None)])
    finally:
        T.tasc_config_set(T.TASC_CFG_STEP_GRAPH, 1)
    for r in runs[1:]:
        assert all((a == b).all() for a, b in zip(r, runs[0]))
    assert (runs[0][0] != greedy).any() and (runs[0][0] != runs[0][1]).any()
    assert (sampled(cfg.k, 0.8, randoms(B, cfg.gen_len, 1)) != runs[0][0]).any()
    # step by step from a rewound session
    T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, cfg.gen_len)
    drafts = torch.zeros((B, cfg.k), dtype=torch.int32, device="cuda")
    for again in range(2):
        T.tasc_session_rewind(rig.session)
        for _ in range(cfg.gen_len):
            T.tasc_draft(rig.ng, rig.session, rig.params(), drafts)
            T.tasc_verify_step_sampled(rig.model, rig.session, drafts, cfg.k, randoms(B, cfg.gen_len), torch.full((B,), 0.8, device="cuda"))
        for b in range(B):
            tokens = T.tasc_session_get_tokens(rig.session, b)[cfg.prompt_len:]
            assert tokens[:cfg.gen_len].tolist() == runs[0][0][b].tolist()


def test_refusals_and_prompts_of_one_token():
    import torch
    rig = rig_of("f32")
    T, B = rig.T, rig.batch
    u = randoms(B, 4)
    drafts = torch.zeros((B, 4), dtype=torch.int32, device="cuda")
    for call in (lambda: T.tasc_session_rewind(rig.session), lambda: T.tasc_verify_step_sampled(rig.model, rig.session, drafts, 4, u)):
        with pytest.raises(T.TascError) as e:
            call()
        assert e.value.status == -4                            # out of order: no prompt yet
    T.tasc_session_prefill(rig.model, rig.session, np.array([1, 2, 3], dtype=np.int32), np.arange(4, dtype=np.int64), 5)
    T.tasc_session_rewind(rig.session)
    T.tasc_verify_step_sampled(rig.model, rig.session, drafts, 4, u)
    assert all(1 < len(T.tasc_session_get_tokens(rig.session, b)) <= 6 for b in range(B))
    small = torch.zeros(256, dtype=torch.uint8, device="cuda")
    for bad in (dict(u=u[:2]), dict(u=u[:, :0]), dict(temperature=torch.zeros(2, device="cuda")), dict(accept_len=drafts), dict(scratch=small), dict(drafts=drafts[:, :2])):
        with pytest.raises(T.TascError):
            T.tasc_verify_step_sampled(**dict(dict(model=rig.model, s=rig.session, drafts=drafts, k=4, u=u), **bad))
    out = torch.zeros((B, 5), dtype=torch.int32, device="cuda")
    with pytest.raises(T.TascError):
        T.tasc_generate_sampled(rig.model, None, rig.session, rig.prompts, rig.prompt_off, 5, rig.params(4), u, out)
