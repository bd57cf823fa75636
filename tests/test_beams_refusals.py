"""More of what the beams' operators refuse, without a GPU: the library's argument checks come before any CUDA call."""
import math
import sysconfig

import torch

from tests.test_beams_host import A8, A8L, AT, EINVAL, Reorder, Select, lib, refused   # noqa: F401


def test_states_that_lie_on_one_another_are_refused(lib):   # noqa: F811
    """Rows that two blocks write while a third reads them: a request or outer stride shorter than a row, a state given twice."""
    base = dict(state=A8(*[AT + 4096 * i for i in range(8)]), outer=A8L(*[2] * 8), outer_stride=A8L(*[256] * 8), request_stride=A8L(*[64] * 8),
                beam_stride=A8L(*[16] * 8), row_bytes=A8L(*[16] * 8), parent=AT, n_states=1, requests=2, beams=4)
    twice = A8(*[AT + 4096 * min(i, 1) for i in range(8)])
    refused(lib, "spd_beam_reorder", Reorder, base, [
        (EINVAL, dict(request_stride=A8L(*[0] * 8))), (EINVAL, dict(outer_stride=A8L(*[0] * 8))), (EINVAL, dict(request_stride=A8L(*[-15] * 8))),
        (EINVAL, dict(outer_stride=A8L(*[8] * 8))), (EINVAL, dict(n_states=2, state=A8(*[AT] * 8))), (EINVAL, dict(n_states=3, state=twice)),
        (0, dict(beams=1, request_stride=A8L(*[0] * 8)))])


def test_an_infinite_power_of_the_length_is_refused(lib):   # noqa: F811
    base = dict(logits=AT, score=AT, new_token=AT, new_parent=AT, new_score=AT, workspace=AT, workspace_bytes=1 << 40, requests=2, beams=4, vocab=100,
                x_dtype=0, eos_id=-1, tau=1.0, request_stride=400, beam_stride=100)
    refused(lib, "spd_beam_select", Select, base, [(EINVAL, dict(alpha=math.inf)), (EINVAL, dict(tau=-math.inf)), (0, dict(requests=0))])


def test_each_python_and_torch_has_a_tensor_module_of_its_own(monkeypatch):
    """The module holds torch's layouts as they were compiled: one that was built for another is not taken for ours."""
    from paper_2405_18400_b200 import beams, build
    path = build.tensors_path()
    assert beams.load_tensors().__file__ == path and torch.__version__ in path and sysconfig.get_config_var("SOABI") in path
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    assert build.tensors_path() != path and build._stale(build.tensors_path())
