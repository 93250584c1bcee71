"""Arguments that are missing, or no tensors, are refused by name (TypeError) both ways through the target-side binding."""
import pytest
import torch

from paper_2609_21858_gb300 import pps

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


def z(*s, dt=torch.bfloat16):
    return torch.zeros(s, dtype=dt, device="cuda")


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def calls():
    q, kc = z(2, 4, 64), z(3, 16, 2, 64)
    yield pps.kv_append, dict(q=q, k=q[:, :2], v=q[:, 2:], pos=i32(0, 1), slot=torch.arange(2, device="cuda"), k_cache=kc,
                              v_cache=kc.clone(), rope=pps.rope_table(16, 64)), (), ("q_norm", "k_norm", "out", "status")
    yield pps.paged_attention, dict(q=q, k_cache=kc, v_cache=kc, pages=i32(0, 1)[None], kv_len=i32(5), q_off=i32(0, 2)), (
        ), ("mask", "out", "lse", "ws", "status")
    yield pps.verify_chain, dict(p_logits=z(2, 50), q_logits=z(1, 50), gamma=1, seq_off=i32(0, 2), node_draft_row=i32(0, -1),
                                 draft_tok=i32(3), u=z(1, dt=torch.float32), noise=z(1, 50, dt=torch.float32) + 1), (
        "gamma",), ("ws", "status")


@pytest.mark.parametrize("named", [False, True])
@pytest.mark.parametrize("which", range(3))
def test_missing_and_foreign_arguments(which, named):
    fn, ok, scalars, optional = list(calls())[which]
    kw = dict(stream=torch.cuda.current_stream()) if named else {}
    fn(**ok, **kw)
    for name in ok:
        if name in scalars:
            continue
        if name != "rope":  # None: no rotation
            with pytest.raises(TypeError, match=name):
                fn(**{**ok, name: None}, **kw)
    for name in list(ok) + list(optional):
        if name in scalars:
            continue
        for x in ([1, 2], 7):
            with pytest.raises(TypeError, match=name):
                fn(**{**ok, name: x}, **kw)
    torch.cuda.synchronize()
