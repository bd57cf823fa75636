"""More of what the beams' operators refuse, without a GPU: the library's argument checks come before any CUDA call."""
import math
import sysconfig

import torch

from tests.test_beams_host import A8, A8L, AT, EINVAL, Append, Attention, Reorder, Select, lib, refused   # noqa: F401


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


ATTENTION = dict(q=AT, k_cache=AT, v_cache=AT, out=AT, prefix_table=AT, prefix_len=AT, own_table=AT, own_len=AT, workspace=AT, workspace_bytes=1 << 40,
                 n=3, b=3, g=1, n_heads=8, n_kv_heads=2, head_dim=64, x_dtype=0, kv_dtype=1, prefix_page=16, prefix_cols=4, own_page=1, own_cols=9, scale=0.125,
                 kc_slot=128, kc_head=64, vc_slot=128, vc_head=64, slots=100)


def test_caches_that_run_backwards_are_refused(lib):   # noqa: F811
    """Their offsets would have read as places that hold nothing."""
    refused(lib, "spd_shared_attention", Attention, ATTENTION, [(EINVAL, dict([(name, -128)])) for name in ("kc_slot", "kc_head", "vc_slot", "vc_head")])


def test_arrays_that_do_not_lie_on_whole_elements_are_refused(lib):   # noqa: F811
    append = dict(q=AT, k=AT, v=AT, q_out=AT, k_cache=AT, v_cache=AT, rope=AT, pos=AT, index=AT, seq=AT, table=AT, status=AT, n=3, n_heads=4, n_kv_heads=2,
                  head_dim=64, rot_dim=64, x_dtype=0, kv_dtype=1, slots=10, page=1, rope_rows=8, table_rows=1, table_cols=1)
    refused(lib, "spd_cache_append", Append, append, [(EINVAL, dict([(name, AT + 2)])) for name in "q k v q_out rope pos index seq table status".split()])
    refused(lib, "spd_cache_append", Append, append, [(EINVAL, dict([(name, AT + 1)])) for name in "k_cache v_cache".split()])
    attention = dict(ATTENTION, lse=AT, q_start=AT, group_start=AT, status=AT)
    refused(lib, "spd_shared_attention", Attention, attention, [(EINVAL, dict([(name, AT + 2)])) for name in
            "q out k_cache v_cache lse q_start group_start prefix_table prefix_len own_table own_len status workspace".split()])
    select = dict(logits=AT, score=AT, length=AT, new_token=AT, new_parent=AT, new_score=AT, new_length=AT, workspace=AT, workspace_bytes=1 << 40, requests=2, beams=4,
                  vocab=100, x_dtype=0, eos_id=-1, tau=1.0, request_stride=400, beam_stride=100)
    refused(lib, "spd_beam_select", Select, select, [(EINVAL, dict([(name, AT + 2)])) for name in
            "logits score length new_token new_parent new_score new_length workspace".split()])
    reorder = dict(state=A8(*[AT] * 8), outer=A8L(*[1] * 8), outer_stride=A8L(*[64] * 8), request_stride=A8L(*[64] * 8), beam_stride=A8L(*[16] * 8),
                   row_bytes=A8L(*[16] * 8), parent=AT, status=AT, n_states=1, requests=2, beams=4)
    refused(lib, "spd_beam_reorder", Reorder, reorder, [(EINVAL, dict(parent=AT + 2)), (EINVAL, dict(status=AT + 1))])
