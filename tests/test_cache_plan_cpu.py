"""Host-side checks of the operators around a kept scene: the plan of a batch's attention, and refusals that need no GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2511_21317_b200 import build
    build.build()


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    out = str(tmp_path_factory.mktemp("plan") / "cache_plan_check")
    subprocess.check_call([gxx, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I/usr/local/cuda/include",
                           os.path.join(ROOT, "tests", "cache_plan_check.cpp"), "-o", out])
    return out


@pytest.mark.parametrize("seed", range(4))
def test_every_key_is_dealt_once(program, seed):
    r = subprocess.run([program, str(seed), "150"], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_null_handles_and_arguments_are_errors():
    from paper_2511_21317_b200 import build, kv_cache as kc
    build.build()
    lib = kc._library()
    v = ctypes.c_int64()
    assert lib.httm_rotary_create(None, None) == -1 and b"null" in lib.httm_last_error(None)
    assert lib.httm_batch_create(None, None) == -1 and b"null" in lib.httm_last_error(None)
    assert lib.httm_rotary_destroy(None) == 0 and lib.httm_batch_destroy(None) == 0
    assert lib.httm_rotary_status(None, ctypes.byref(v)) == -1 and lib.httm_batch_status(None, ctypes.byref(v)) == -1
    assert lib.httm_norm_rotate(None, 0, 1, None, None, None, None) == -1
    assert lib.httm_norm_rotate_backward(None, 0, 1, None, None, None, None) == -1
    assert lib.httm_batch_set(None, 0, None, None, None, 0, None, 0, None) == -1
    null = kc._Tensor(None, 0, 0)
    pages = kc._Pages(None, 0, 0, 0)
    assert lib.httm_cache_append(None, 0, pages, pages, null, null, None, None, None, None, None) == -1
    assert lib.httm_cache_attention(None, 0, pages, pages, null, null, 1.0, None) == -1


@pytest.mark.parametrize("kw,code", [(dict(head_dim=48), -2), (dict(norm="layer", axes=3), -1), (dict(rotated_dim=20), -1), (dict(rotated_dim=72), -1),
                                     (dict(axes=2, rotated_dim=24), -1), (dict(n_positions=0), -1), (dict(eps=-1.0), -1), (dict(base=0.0), -1),
                                     (dict(device=99), -1), (dict(norm="batch"), -1), (dict(frequencies=[1.0]), -1)])
def test_rotary_refuses(kw, code):
    from paper_2511_21317_b200 import binding, kv_cache as kc
    base = dict(head_dim=64, n_positions=8)
    base.update(kw)
    with pytest.raises(binding.HttmError) as e:
        kc.Rotary(**base)
    assert e.value.code == code


@pytest.mark.parametrize("kw,code", [(dict(heads=6, kv_heads=4), -1), (dict(heads=129, kv_heads=1), -2), (dict(head_dim=96), -2), (dict(page_size=24), -2),
                                     (dict(page_size=8), -2), (dict(n_pages=0), -1), (dict(n_pages=1 << 30), -1), (dict(kv_heads=0), -1), (dict(device=99), -1)])
def test_batch_refuses(kw, code):
    from paper_2511_21317_b200 import binding, kv_cache as kc
    base = dict(heads=4, kv_heads=4, head_dim=64, page_size=16, n_pages=8)
    base.update(kw)
    with pytest.raises(binding.HttmError) as e:
        kc.CacheBatch(**base)
    assert e.value.code == code
