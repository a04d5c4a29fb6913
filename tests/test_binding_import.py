"""The binding on a machine, or with a torch, that has no GPU support: it imports, checks arguments and refuses tensors that are not on a GPU."""
import subprocess
import sys

import pytest
import torch

from paper_2605_19726_amd import binding as bd
from paper_2605_19726_amd import build


def test_a_torch_without_gpu_support_imports_it_and_gets_its_checks():
    code = ("import torch\n"
            "for name in ('_cuda_getCurrentRawStream', '_cuda_getDevice'):\n"
            "    if hasattr(torch._C, name): delattr(torch._C, name)\n"
            "from paper_2605_19726_amd import binding as bd\n"
            "x = torch.zeros(2, 1, 16, 64)\n"
            "assert bd.PagedCache(x, x).page == 16 and bd.params(128).block == 128\n"
            "try: bd.PagedCache(x, x.half())\n"
            "except ValueError: print('checked')\n")
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=build.ROOT)
    assert done.returncode == 0 and done.stdout.strip() == "checked", done.stderr


def test_the_public_ways_stand_in_for_the_short_ones(monkeypatch):
    import importlib.util
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    spec = importlib.util.spec_from_file_location("binding_again", bd.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)

    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: Stream if device == 3 else None)
    assert again._raw_stream(3) == 77 and again._current_device is torch.cuda.current_device


def test_tensors_that_are_not_on_a_gpu_are_refused():
    x, ints = torch.zeros(1, 2, 200, 64), lambda *shape: torch.zeros(shape, dtype=torch.int32)
    cache = bd.PagedCache(x, x)
    rows, q, table = torch.zeros(3, 2, 64), torch.zeros(3, 4, 64), ints(3, 2)
    for call in (lambda: bd.basa_norm_sort(x, 128), lambda: bd.ba_att(x, x, x), lambda: bd.basa_downsample(x, 128),
                 lambda: bd.basa_page_tables(ints(3), ints(3), table, ints(9), 16, 5),
                 lambda: bd.basa_cache_append(rows, rows, torch.zeros(3, dtype=torch.int64), cache),
                 lambda: bd.basa_cache_gather(cache, table, ints(4), 5), lambda: bd.basa_decode_attn(q, cache, table, ints(3))):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
