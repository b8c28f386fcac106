"""What the operators on pages write to in the caller's tensors counts as a change in place, for autograd; nothing else does."""
import pytest

import paper_2510_15312_b200 as pkg
from test_gpu_paged import calls, i32

pytestmark = pytest.mark.gpu


def outputs(name, a, kw):
    """Outputs that may be given, by keyword, and the tensors behind them."""
    import torch
    made = getattr(pkg, name)(*a, **kw)
    if name in ("paged_slots", "verify_sampled"):
        out = tuple(None if x is None else x.clone() for x in made)
        return dict(out=out), [x for x in out if x is not None]
    if made is None:
        return {}, []
    out = torch.empty_like(made, memory_format=torch.contiguous_format)
    status = i32([0])
    return (dict(q_out=out), [out]) if name == "rope_append" else (dict(out=out, status=status), [out, status])


@pytest.mark.parametrize("which", range(6))
@pytest.mark.parametrize("mode", ["plain", "inference"])
def test_versions(which, mode):
    import torch
    with torch.inference_mode(mode == "inference"):
        name, a, kw = calls()[which]
        more, out = outputs(name, a, kw)
        changed = [a[2]] if name == "paged_slots" else [kw["k_pages"], kw["v_pages"]] if "k_pages" in kw else list(a[5:7]) if name == "rope_append" else []
    given = [x for x in (*a, *kw.values(), *out) if torch.is_tensor(x)]
    if mode == "inference":   # tensors without a counter are taken as they are
        assert all(x.is_inference() for x in given)
        getattr(pkg, name)(*a, **kw, **more)
        return
    before = [x._version for x in given]
    getattr(pkg, name)(*a, **kw, **more)
    for x, v in zip(given, before):
        written = any(x is y for y in changed + out)
        assert (x._version > v) == written, (name, x.shape)


def test_a_saved_tensor_that_was_written_to_is_noticed():
    import torch
    name, a, kw = calls()[2]
    x = torch.ones(kw["k_pages"].shape, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    pages = x * 2
    loss = (pages * pages).sum()             # keeps the pages for its gradient
    pkg.rope_append(*a, **{**kw, "k_pages": pages.detach()})
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()


def test_refused_calls_change_nothing():
    import torch
    name, a, kw = calls()[0]
    versions = [x._version for x in a if torch.is_tensor(x)]
    with pytest.raises(pkg.SdvError):
        pkg.paged_slots(*a[:6], 0, 6)
    assert versions == [x._version for x in a if torch.is_tensor(x)]
