"""Operators of k real drafts behind one prompt: paged append, shared-prefix attention, beam selection, reordering.

Marshalling only, as binding.py: the arithmetic is the library's (include/spd.h says what each operator computes and refuses), the
tensors' checks and the argument structs are a compiled module's (csrc/spd_tensors.cpp: in Python they cost several times what
a timestep's calls take on the device).  Every call is enqueued on the current stream of its tensors' device and allocates nothing there
but its outputs (and the attention's and the selection's workspace where none is passed); tensors may be views with strides as long as
their last dimension is contiguous.  Tensors that do not fit one another raise ValueError, what the library refuses SpdError.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from typing import Optional, Sequence, Union

import torch

from . import build as _build
from .binding import _check, load_library

_PAIRS = {"adjacent": 0, "halves": 1}
_tensors = None


def load_tensors():
    """The module that takes tensors to the operators, built first when its source is newer or none is there for this Python and torch, tied
    to the loaded library."""
    global _tensors
    if _tensors is None:
        library, path = load_library(), _build.tensors_path()
        try:
            _build.build_tensors()
        except Exception as exc:  # no compiler on this machine: the prebuilt module must be there
            if not os.path.exists(path):
                raise RuntimeError("%s is missing and could not be built: %s" % (os.path.basename(path), exc)) from exc
        spec = importlib.util.spec_from_file_location(__package__ + "._spd_tensors", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.bind(*[C.cast(getattr(library, name), C.c_void_p).value for name in (
            "spd_cache_append", "spd_shared_attention", "spd_shared_attention_bytes", "spd_beam_select", "spd_beam_select_bytes", "spd_beam_reorder")],
                    _check, torch.OutOfMemoryError)
        _tensors = module
    return _tensors


def spd_rope_table(positions: int, rot_dim: int, theta: float = 10000.0, device: Union[str, torch.device] = "cuda:0") -> torch.Tensor:
    """cos and sin of position * theta^(-2 p / rot_dim), [positions, rot_dim / 2, 2] float32, worked out in 64 bits."""
    inv = theta ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return torch.stack([angle.cos(), angle.sin()], -1).to(torch.float32).contiguous().to(device)


def spd_cache_append(k: Optional[torch.Tensor], v: Optional[torch.Tensor], k_cache: Optional[torch.Tensor], v_cache: Optional[torch.Tensor],
                     pos: torch.Tensor, rope: Optional[torch.Tensor], *, q: Optional[torch.Tensor] = None,
                     q_out: Optional[torch.Tensor] = None, index: Optional[torch.Tensor] = None, seq: Optional[torch.Tensor] = None,
                     table: Optional[torch.Tensor] = None, page: int = 1, pairs: str = "adjacent",
                     status: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Stores k and v [n, kv_heads, dim] into the caches [slots, kv_heads, dim], rotated (k, and q if given) by the angles of
    `pos` [n] in `rope` (spd_rope_table; None: no rotation).  Token i goes to place index[i] (default pos[i]) of row seq[i]
    (default i) of `table` [sequences, pages], or to slot index[i] without a table.  Returns the rotated queries (a new tensor, or
    q_out), None without q."""
    return (_tensors or load_tensors()).cache_append(k, v, k_cache, v_cache, pos, rope, q, q_out, index, seq, table, page, _PAIRS.get(pairs, -1), status)


def spd_shared_attention_workspace(q: torch.Tensor, k_cache: torch.Tensor, own_table: torch.Tensor,
                                   prefix_table: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Workspace for calls with as many query rows, sequences and prefixes as these tensors have, or fewer; to be kept between calls."""
    types = {torch.float32: 0, torch.bfloat16: 1}
    with torch.cuda.device(q.device):
        size = (_tensors or load_tensors()).shared_attention_bytes(
            q.shape[0], own_table.shape[0], 0 if prefix_table is None else prefix_table.shape[0], q.shape[1], k_cache.shape[1], q.shape[2],
            types.get(q.dtype, -1), types.get(k_cache.dtype, -1))
    return torch.empty(size, dtype=torch.uint8, device=q.device)


def spd_shared_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, own_table: torch.Tensor, own_len: torch.Tensor, *,
                         own_page: int = 1, prefix_table: Optional[torch.Tensor] = None, prefix_len: Optional[torch.Tensor] = None,
                         prefix_page: int = 1, group_start: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
                         scale: Optional[float] = None, out: Optional[torch.Tensor] = None, return_lse: bool = False,
                         workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Attention of q [n, heads, dim] over the shared prefixes and the sequences' own tokens, whose keys and values lie in the caches
    [slots, kv_heads, dim].  Sequences are the rows of own_table [b, pages] (own_len [b] places in use), prefixes those of
    prefix_table [g, pages] (prefix_len [g]); group j is sequences group_start[j] .. group_start[j + 1] (needed when g > 1).  One query
    row per sequence, or rows q_start[s] .. q_start[s + 1] as sequence s's last tokens.  scale: 1 / sqrt(dim) by default.  Returns
    out [n, heads, dim], with return_lse also the log-sum-exp [n, heads]."""
    return (_tensors or load_tensors()).shared_attention(q, k_cache, v_cache, own_table, own_len, own_page, prefix_table, prefix_len, prefix_page,
                                                         group_start, q_start, scale, out, return_lse, workspace, status)


def spd_beam_select_workspace(logits: torch.Tensor) -> torch.Tensor:
    """Workspace for selections of this shape and type, or of fewer requests; to be kept between calls (its counters come zeroed, and calls leave them so)."""
    return torch.zeros((_tensors or load_tensors()).beam_select_bytes(logits), dtype=torch.uint8, device=logits.device)


def spd_beam_select(logits: torch.Tensor, score: torch.Tensor, length: Optional[torch.Tensor] = None, finished: Optional[torch.Tensor] = None, *,
                    eos_id: int = -1, tau: float = 1.0, length_alpha: float = 0.0, workspace: Optional[torch.Tensor] = None):
    """The best beams of logits [requests, beams, vocab] behind beams of log-probability `score` [requests, beams] (float32; minus infinity:
    not in use), `length` (int32, zeros if None) and `finished` (bool, none if None).  Returns (token, parent, score, length,
    finished), each [requests, beams], best first."""
    if workspace is None:
        workspace = spd_beam_select_workspace(logits)
    return (_tensors or load_tensors()).beam_select(logits, score, length, finished, eos_id, tau, length_alpha, workspace)


def spd_beam_reorder(states: Union[torch.Tensor, Sequence[torch.Tensor]], parent: torch.Tensor, *, dim: int = 0,
                     status: Optional[torch.Tensor] = None) -> None:
    """In place: beam j of request r becomes what beam parent[r, j] was, in every state.  A state has requests and beams as its
    dimensions `dim` and `dim` + 1; those behind are contiguous (a view of the first steps will do), those in front have one stride.  No element may
    be there twice, in a state or in two of them."""
    states = (states,) if isinstance(states, torch.Tensor) else tuple(states)
    (_tensors or load_tensors()).beam_reorder(states, parent, dim, status)
