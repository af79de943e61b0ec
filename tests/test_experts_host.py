"""Operators of a mixture-of-experts layer: declarations, exports and refusals, all of which come before any
launch and need no GPU."""
import os
import re

import pytest

from paper_1705_01598_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                       # a stand-in for device memory: never looked at, since every call here is refused


def test_library_exports_every_declared_call():
    text = open(os.path.join(ROOT, "include", "tperm_experts.h")).read()
    declared = re.findall(r"\btperm_status_t (tperm_[a-z_]+)\(", text)
    assert declared == B.EXPERT_EXPORTS
    for name in declared:
        assert hasattr(B.lib(), name), name
    assert f"#define TPERM_EXPERTS_MAX {B.EXPERTS_MAX}" in text and f"#define TPERM_SLOTS_MAX {B.SLOTS_MAX}" in text
    assert f"#define TPERM_EXPERT_SORT_ONE_BLOCK {B.EXPERT_SORT_ONE_BLOCK}" in text and B.WIDTH_MAX == 1 << 20


# Arguments that are accepted by the checks up to the one that a test changes.  Arrays lie 1 GiB apart.
def _at(i):
    return P + (i << 30)


CALLS = {
    "tperm_expert_sort": dict(expert_ptr=_at(0), tokens=4, slots=2, experts=3, offsets_ptr=_at(1), source_ptr=_at(2), place_ptr=_at(3)),
    "tperm_expert_gather": dict(x_ptr=_at(0), x_stride=16, source_ptr=_at(1), offsets_ptr=_at(2), weights_ptr=_at(3), out_ptr=_at(4), out_stride=16,
                                tokens=4, slots=2, experts=3, width=16, dtype=B.TYPE_BF16),
    "tperm_expert_combine": dict(rows_ptr=_at(0), rows_stride=16, place_ptr=_at(1), offsets_ptr=_at(2), weights_ptr=_at(3), out_ptr=_at(4), out_stride=16,
                                 tokens=4, slots=2, experts=3, width=16, dtype=B.TYPE_BF16),
    "tperm_expert_combine_backward": dict(grad_ptr=_at(0), grad_stride=16, rows_ptr=_at(1), rows_stride=16, place_ptr=_at(2), offsets_ptr=_at(3),
                                          weights_ptr=_at(4), grad_rows_ptr=_at(5), grad_rows_stride=16, grad_weights_ptr=_at(6), tokens=4, slots=2,
                                          experts=3, width=16, dtype=B.TYPE_BF16),
    "tperm_expert_product": dict(x_ptr=_at(0), x_stride=16, x_rows=4, source_ptr=_at(1), slots=2, offsets_ptr=_at(2), w_ptr=_at(3), w_k_first=True,
                                 out_ptr=_at(4), out_stride=24, rows=8, experts=3, k=16, n=24, dtype=B.TYPE_BF16),
    "tperm_expert_weight_gradient": dict(x_ptr=_at(0), x_stride=16, x_scales_ptr=_at(1), x_rows=4, source_ptr=_at(2), slots=2, grad_ptr=_at(3),
                                         grad_stride=24, offsets_ptr=_at(4), out_ptr=_at(5), out_dtype=B.TYPE_F32, w_k_first=False, accumulate=False,
                                         rows=8, experts=3, k=16, n=24, dtype=B.TYPE_BF16),
    "tperm_checkpoint_store": dict(x_ptr=_at(0), x_stride=16, codes_ptr=_at(1), scales_ptr=_at(2), rows=4, width=16, dtype=B.TYPE_BF16),
    "tperm_checkpoint_load": dict(codes_ptr=_at(0), scales_ptr=_at(1), out_ptr=_at(2), out_stride=16, rows=4, width=16, dtype=B.TYPE_BF16),
    "tperm_gated_forward": dict(gates_ptr=_at(0), gates_stride=32, out_ptr=_at(1), out_stride=16, codes_ptr=_at(2), scales_ptr=_at(3), rows=4, width=16,
                                dtype=B.TYPE_BF16),
    "tperm_gated_backward": dict(grad_ptr=_at(0), grad_stride=16, codes_ptr=_at(1), scales_ptr=_at(2), grad_gates_ptr=_at(3), grad_gates_stride=32,
                                 out_ptr=_at(4), out_stride=16, rows=4, width=16, dtype=B.TYPE_BF16),
}


def _refused(name, status, **changes):
    with pytest.raises(B.TpermError) as e:
        getattr(B, name)(**{**CALLS[name], **changes})
    assert e.value.status == status, (name, changes, str(e.value))


def _pointers(name):
    return [k for k in CALLS[name] if k.endswith("_ptr")]


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_pointers_are_refused(name):
    for k in _pointers(name):
        optional = (k == "weights_ptr" and name != "tperm_expert_combine_backward") or (k == "x_scales_ptr") \
            or (k == "out_ptr" and name == "tperm_gated_backward") \
            or (k == "source_ptr" and name in ("tperm_expert_product", "tperm_expert_weight_gradient"))
        if not optional:
            _refused(name, B.ERR_NULL, **{k: None})


@pytest.mark.parametrize("name", sorted(CALLS))
def test_sizes_and_strides_outside_their_limits_are_refused(name):
    a = CALLS[name]
    bad = {"slots": (0, B.SLOTS_MAX + 1, -1), "experts": (0, B.EXPERTS_MAX + 1, -3), "width": (0, -1, B.WIDTH_MAX + 1), "k": (0, B.WIDTH_MAX + 1),
           "n": (0, -5, B.WIDTH_MAX + 1), "tokens": (-1,), "rows": (-1,), "x_rows": (-1,)}
    for k, values in bad.items():
        for v in values if k in a else ():
            _refused(name, B.ERR_DIMS, **{k: v})
    for k in a:
        if k.endswith("_stride") and not (name == "tperm_expert_weight_gradient" and k == "x_stride"):
            _refused(name, B.ERR_DIMS, **{k: a[k] - 1})
            _refused(name, B.ERR_DIMS, **{k: (1 << 28) + 1})
    if "tokens" in a:
        _refused(name, B.ERR_TOO_LARGE, tokens=1 << 30)       # 2 slots: 2^31 rows
        _refused(name, B.ERR_TOO_LARGE, tokens=1 << 62)
    if "rows" in a:
        _refused(name, B.ERR_TOO_LARGE, rows=1 << 31)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_types_alignment_and_overlap(name):
    a = CALLS[name]
    if "dtype" in a:
        for t in (-1, 3, 100):
            _refused(name, B.ERR_ELEM_SIZE, dtype=t)
    if "out_dtype" in a:
        _refused(name, B.ERR_ELEM_SIZE, out_dtype=7)
    bytes_only = {"codes_ptr", "scales_ptr", "x_scales_ptr"} | ({"x_ptr"} if name == "tperm_expert_weight_gradient" else set())
    for k in _pointers(name):
        if k not in bytes_only:
            _refused(name, B.ERR_ALIGN, **{k: a[k] + 1})
    outputs = {"tperm_expert_sort": ["offsets_ptr", "source_ptr", "place_ptr"], "tperm_expert_combine_backward": ["grad_rows_ptr", "grad_weights_ptr"],
               "tperm_checkpoint_store": ["codes_ptr", "scales_ptr"], "tperm_gated_forward": ["out_ptr", "codes_ptr", "scales_ptr"],
               "tperm_gated_backward": ["grad_gates_ptr", "out_ptr"]}.get(name, ["out_ptr"])
    for o in outputs:
        for k in _pointers(name):
            if k != o:
                _refused(name, B.ERR_ALIAS, **{o: a[k]})


def test_sort_asks_for_its_workspace():
    many = dict(CALLS["tperm_expert_sort"], tokens=B.EXPERT_SORT_ONE_BLOCK, slots=2)
    need = B.expert_sort_workspace_bytes(2 * B.EXPERT_SORT_ONE_BLOCK, 3)
    assert need == 128 * 4 * 4 and B.expert_sort_workspace_bytes(B.EXPERT_SORT_ONE_BLOCK, 3) == 0
    for ws, status in ((dict(), B.ERR_NULL), (dict(workspace_ptr=_at(5), workspace_bytes=need - 1), B.ERR_TOO_LARGE),
                       (dict(workspace_ptr=_at(5) + 2, workspace_bytes=need), B.ERR_ALIGN), (dict(workspace_ptr=_at(0), workspace_bytes=need), B.ERR_ALIAS)):
        with pytest.raises(B.TpermError) as e:
            B.tperm_expert_sort(**{**many, **ws})
        assert e.value.status == status


def test_products_state_their_sizes():
    big = 1 << 20
    _refused("tperm_expert_product", B.ERR_TOO_LARGE, k=big, n=big // 256, x_stride=big, out_stride=big)          # a matrix of 8 GiB
    _refused("tperm_expert_product", B.ERR_TOO_LARGE, x_stride=1 << 28, x_rows=16)                                # a gathered x of 8 GiB
    _refused("tperm_expert_product", B.ERR_DIMS, source_ptr=None, x_rows=7)                                       # fewer rows than the order has
    _refused("tperm_expert_weight_gradient", B.ERR_TOO_LARGE, k=big, n=big // 256, grad_stride=big)
    _refused("tperm_expert_weight_gradient", B.ERR_DIMS, x_scales_ptr=None, x_stride=15)
    _refused("tperm_gated_forward", B.ERR_NULL, codes_ptr=None)


def test_nothing_to_do_is_no_launch():
    for name in CALLS:
        if "tokens" in CALLS[name] and name != "tperm_expert_sort":
            getattr(B, name)(**{**CALLS[name], **{k: None for k in _pointers(name)}, "tokens": 0})
    B.tperm_expert_product(**{**CALLS["tperm_expert_product"], "rows": 0, "x_ptr": None, "x_rows": 0})
    for name in ("tperm_checkpoint_store", "tperm_checkpoint_load", "tperm_gated_backward"):
        getattr(B, name)(**{**CALLS[name], **{k: None for k in _pointers(name)}, "rows": 0})


def test_arguments_of_other_types():
    a = dict(CALLS["tperm_checkpoint_store"])
    with pytest.raises(TypeError):
        B.tperm_checkpoint_store(**{**a, "x_ptr": 1.5})
    with pytest.raises(TypeError):
        B.tperm_checkpoint_store(**{**a, "rows": "4"[:0] or None})
    with pytest.raises(OverflowError):
        B.tperm_checkpoint_store(**{**a, "dtype": 1 << 32})          # not taken for type 0
    with pytest.raises(TypeError):
        B._calls().checkpoint_store(1, 2, 3)
