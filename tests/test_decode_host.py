"""Router, matrices in 4 bits and the layer for a few tokens: declarations, exports and refusals, all of which come
before any launch and need no GPU."""
import os
import re

import pytest

from paper_1705_01598_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _at(i):
    """Stand-ins for device memory, 1 GiB apart: never looked at, since every call here is refused."""
    return (1 << 20) + (i << 30)


CALLS = {
    "tperm_expert_route": dict(scores_ptr=_at(0), scores_stride=6, expert_ptr=_at(1), weights_ptr=_at(2), tokens=4, slots=2, experts=6, over_all=False,
                               dtype=B.TYPE_BF16),
    "tperm_expert_route_backward": dict(grad_weights_ptr=_at(0), scores_ptr=_at(1), scores_stride=6, expert_ptr=_at(2), weights_ptr=_at(3),
                                        grad_scores_ptr=_at(4), grad_scores_stride=6, tokens=4, slots=2, experts=6, over_all=True, dtype=B.TYPE_BF16),
    "tperm_four_bit_store": dict(x_ptr=_at(0), x_stride=40, codes_ptr=_at(1), scales_ptr=_at(2), rows=4, width=40, dtype=B.TYPE_BF16),
    "tperm_four_bit_load": dict(codes_ptr=_at(0), scales_ptr=_at(1), out_ptr=_at(2), out_stride=40, rows=4, width=40, dtype=B.TYPE_BF16),
    "tperm_four_bit_product": dict(x_ptr=_at(0), x_stride=40, codes_ptr=_at(1), scales_ptr=_at(2), out_ptr=_at(3), out_stride=24, rows=4, k=40, n=24,
                                   dtype=B.TYPE_BF16),
    "tperm_expert_few": dict(x_ptr=_at(0), x_stride=40, expert_ptr=_at(1), weights_ptr=_at(2), w_in_ptr=_at(3), w_in_scales_ptr=_at(4), w_out_ptr=_at(5),
                             w_out_scales_ptr=_at(6), out_ptr=_at(7), out_stride=40, workspace_ptr=_at(8), workspace_bytes=1 << 20, tokens=4, slots=2,
                             experts=6, width=40, hidden=24, dtype=B.TYPE_BF16),
}
OUTPUTS = {"tperm_expert_route": ["expert_ptr", "weights_ptr"], "tperm_expert_route_backward": ["grad_scores_ptr"], "tperm_four_bit_store": ["codes_ptr", "scales_ptr"],
           "tperm_expert_few": ["out_ptr", "workspace_ptr"]}


def _refused(name, status, **changes):
    with pytest.raises(B.TpermError) as e:
        getattr(B, name)(**{**CALLS[name], **changes})
    assert e.value.status == status, (name, changes, str(e.value))


def _pointers(name):
    return [k for k in CALLS[name] if k.endswith("_ptr")]


def test_library_exports_every_declared_call():
    text = open(os.path.join(ROOT, "include", "tperm_decode.h")).read()
    assert re.findall(r"\btperm_status_t (tperm_[a-z_]+)\(", text) == B.DECODE_EXPORTS
    for name in B.DECODE_EXPORTS + ["tperm_expert_few_workspace"]:
        assert hasattr(B.lib(), name), name
    assert f"#define TPERM_FEW_TOKENS {B.FEW_TOKENS}\n" in text


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_pointers_are_refused(name):
    for k in _pointers(name):
        if not (name == "tperm_expert_few" and k == "weights_ptr"):
            _refused(name, B.ERR_NULL, **{k: None})


@pytest.mark.parametrize("name", sorted(CALLS))
def test_sizes_and_strides_outside_their_limits_are_refused(name):
    a = CALLS[name]
    bad = {"slots": (0, B.SLOTS_MAX + 1, -1), "experts": (0, B.EXPERTS_MAX + 1, -3), "width": (0, -1, B.WIDTH_MAX + 1), "k": (0, B.WIDTH_MAX + 1),
           "n": (0, -5, B.WIDTH_MAX + 1), "tokens": (-1,), "rows": (-1,), "hidden": (0, -1, B.WIDTH_MAX // 2 + 1, 1 << 62)}
    for k, values in bad.items():
        for v in values if k in a else ():
            _refused(name, B.ERR_DIMS, **{k: v})
    for k in a:
        if k.endswith("_stride"):
            _refused(name, B.ERR_DIMS, **{k: a[k] - 1})
            _refused(name, B.ERR_DIMS, **{k: (1 << 28) + 1})
    if name == "tperm_expert_few":
        _refused(name, B.ERR_DIMS, tokens=B.FEW_TOKENS + 1)
    if "tokens" in a:
        for tokens in (1 << 30, 1 << 62):           # 2 slots: 2^31 rows
            _refused(name, B.ERR_TOO_LARGE, tokens=tokens)
    if "rows" in a:
        _refused(name, B.ERR_TOO_LARGE, rows=1 << 31)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_types_alignment_and_overlap(name):
    a = CALLS[name]
    for t in (-1, 3, 100):
        _refused(name, B.ERR_ELEM_SIZE, dtype=t)
    for k in _pointers(name):
        if not k.endswith("scales_ptr"):
            _refused(name, B.ERR_ALIGN, **{k: a[k] + 1})
        if k in ("codes_ptr", "w_in_ptr", "w_out_ptr", "workspace_ptr"):
            _refused(name, B.ERR_ALIGN, **{k: a[k] + 8})
    for o in OUTPUTS.get(name, ["out_ptr"]):
        for k in _pointers(name):
            if k != o:
                _refused(name, B.ERR_ALIAS, **{o: a[k]})


def test_scores_that_are_not_read_may_be_missing_or_anything():
    """The form without over_all: what is refused is another argument."""
    for scores in (None, _at(1) + 1, CALLS["tperm_expert_route_backward"]["grad_scores_ptr"]):
        _refused("tperm_expert_route_backward", B.ERR_NULL, over_all=False, scores_ptr=scores, scores_stride=0, expert_ptr=None)


def test_matrices_are_of_one_kind_and_of_their_size():
    name = "tperm_expert_few"
    _refused(name, B.ERR_NULL, w_in_scales_ptr=None)
    _refused(name, B.ERR_NULL, w_out_scales_ptr=None)
    plain = dict(w_in_scales_ptr=None, w_out_scales_ptr=None)
    _refused(name, B.ERR_ALIGN, **plain, w_in_ptr=_at(3) + 1)
    big = dict(width=1 << 20, x_stride=1 << 20, out_stride=1 << 20)
    _refused(name, B.ERR_TOO_LARGE, **big, **plain, hidden=1 << 10)        # 2^31 elements of 2 bytes in one w_in
    _refused(name, B.ERR_TOO_LARGE, **big, hidden=1 << 12)                 # 2^33 in 4 bits
    _refused("tperm_four_bit_product", B.ERR_TOO_LARGE, k=1 << 20, n=1 << 13, x_stride=1 << 20, out_stride=1 << 13)


def test_workspace_is_asked_for():
    a = CALLS["tperm_expert_few"]
    need = B.expert_few_workspace_bytes(4, 2, 6, 40, 24, B.TYPE_BF16, True)
    assert 0 < need < 1 << 20
    _refused("tperm_expert_few", B.ERR_TOO_LARGE, workspace_bytes=need - 1)
    assert a["workspace_bytes"] >= need
    for bad in ((0, 2, 6, 40, 24), (65, 2, 6, 40, 24), (4, 0, 6, 40, 24), (4, 2, 1025, 40, 24), (4, 2, 6, 0, 24), (4, 2, 6, 40, 1 << 20)):
        assert B.expert_few_workspace_bytes(*bad, B.TYPE_BF16) == 0
    assert B.expert_few_workspace_bytes(4, 2, 6, 40, 24, 3) == 0


def test_nothing_to_do_is_no_launch():
    for name, a in CALLS.items():
        k = "tokens" if "tokens" in a else "rows"
        nothing = {p: None for p in _pointers(name)}
        getattr(B, name)(**{**a, **nothing, k: 0})


def test_arguments_of_other_types():
    a = CALLS["tperm_four_bit_store"]
    with pytest.raises(TypeError):
        B.tperm_four_bit_store(**{**a, "x_ptr": 1.5})
    with pytest.raises(OverflowError):
        B.tperm_four_bit_store(**{**a, "dtype": 1 << 32})
    with pytest.raises(TypeError):
        B._calls().expert_route(1, 2, 3)
    with pytest.raises(TypeError):
        B._calls().bind_decode(1, 2, 3)
