"""Where a sampled step's time is booked: its acceptance under "accept" in every kernel family, once a step."""
import numpy as np
import pytest

from test_gpu_sampled_decoding import MODELS, randoms, rig_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name, kernel", [(name, 1) for name in MODELS] + [("persistent", 0)])
def test_acceptance_of_sampled_steps(name, kernel):
    import torch
    rig = rig_of(name)
    T, B, k = rig.T, rig.batch, rig.cfg.k
    u = randoms(B, 8)
    T.tasc_session_prefill(rig.model, rig.session, rig.prompts, rig.prompt_off, 8)
    drafts = torch.zeros((B, k), dtype=torch.int32, device="cuda")
    try:
        T.tasc_config_set(T.TASC_CFG_SMALL_KERNEL, kernel)
        T.tasc_profile_enable(["accept", "layers"])
        for _ in range(3):
            T.tasc_verify_step_sampled(rig.model, rig.session, drafts, k, u)
        torch.cuda.synchronize()
        got = T.tasc_profile_read()
    finally:
        T.tasc_profile_enable([])
        T.tasc_config_set(T.TASC_CFG_SMALL_KERNEL, 1)
    assert got["accept"][1] == 3 and got["accept"][0] > 0
    assert got.get("layers", (0, 0))[1] == (3 if name == "persistent" else 0)
