"""The linear calls refuse workspaces that kernels cannot write anywhere in: on the host, or not in one piece."""
import pytest
import torch

from tests.test_paged_numerics import DEV, WORKSPACES, _on_gpu, launches  # noqa: F401 (a fixture)


@pytest.mark.parametrize("what", sorted(WORKSPACES))
def test_linear_calls_refuse_a_workspace_that_is_not_one_piece_on_the_gpu(launches, what):
    import paper_2505_15909_amd as rtn
    A, W, q, s, C = _on_gpu(2, 256), _on_gpu(64, 256), _on_gpu(64 * 128, dtype=torch.uint8), _on_gpu(64, 2), _on_gpu(2, 64)
    modules = [{"A": A, "qweight": q, "scales": s, "bits": 4, "group_size": 128, "C": C}]
    calls = {"rtn_linear_ex": lambda w: rtn.rtn_linear(A, q, s, 4, 128, out=C, workspace=w), "rtn_linear_asym": lambda w: rtn.rtn_linear_asym(A, q, s, s, 4, 128, out=C, workspace=w),
             "rtn_gemm_fp16": lambda w: rtn.rtn_gemm_fp16(A, W, out=C, workspace=w), "rtn_linear_dense": lambda w: rtn.rtn_linear_dense(A, q, s, 4, 128, W, out=C, workspace=w),
             "rtn_layer_forward": lambda w: rtn.rtn_layer_forward(modules, w), "rtn_grouped_forward": lambda w: rtn.rtn_grouped_forward(modules, w)}
    for call in calls.values():
        with pytest.raises(ValueError, match="workspace"):
            call(WORKSPACES[what](_on_gpu))
    with pytest.raises(ValueError, match="w_tmp"):
        rtn.rtn_linear_dense(A, q, s, 4, 128, WORKSPACES[what](_on_gpu), out=C)
    assert not launches
    for call in calls.values():
        call(_on_gpu(1 << 16, dtype=torch.uint8))
    assert [name for name, _ in launches] == list(calls)


@pytest.mark.gpu
@pytest.mark.parametrize("what", sorted(WORKSPACES))
def test_native_linear_calls_leave_such_a_workspace_to_be_refused(rtn, what):
    ws = WORKSPACES[what](lambda *n, dtype: torch.zeros(*n, dtype=dtype, device=DEV))
    A, W = torch.randn(2, 512, device=DEV).half(), torch.randn(64, 512, device=DEV).half()
    C = torch.empty(2, 64, dtype=torch.float16, device=DEV)
    with pytest.raises(ValueError, match="workspace"):
        rtn.rtn_linear(A, *rtn.rtn_quantize(W, 4, 128), 4, 128, out=C, workspace=ws)
    with pytest.raises(ValueError, match="workspace"):
        rtn.rtn_linear_asym(A, *rtn.rtn_quantize_asym(W, 4, 128), 4, 128, out=C, workspace=ws)
