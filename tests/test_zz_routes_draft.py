"""Which kernel the calls on drafted tokens launch (names from torch's profiler, see test_zz_routes.py): the shapes that the tests of their numbers run are
those of every form."""
import pytest

from test_gpu_draft_projection import FORMS, project
from test_zz_routes import _kernels_of, _need_256_cus

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,H,Hq,Hkv,D,B,T", FORMS)
def test_which_form_a_projection_takes(form, H, Hq, Hkv, D, B, T):
    _need_256_cus()
    pc, x, w, parents, pos0, _ = project(form, H, Hq, Hkv, D, B, T)
    names = [n for n in _kernels_of(lambda: pc.percache_qkv_rope_draft(x, w, pos0, parents=parents)) if "qkv" in n]
    kind, _, blocks = form.partition(" ")
    want = {"few": "qkv_rope_few_kernel", "deep": f"qkv_rope_kernelILi{D}ELi2ELb0ELb0ELb1E", "wide": f"qkv_rope_kernelILi{D}ELi{blocks}ELb0ELb1ELb0E",
            "plain": f"qkv_rope_kernelILi{D}ELi{blocks}ELb0ELb0ELb0E"}[kind]
    assert len(names) == 1 and want in names[0], names
    pc.close()
