"""The compiled part of the binding: what it refuses before the library is called, and that the library offers every call of the header."""
import os
import re

import pytest
import torch

from paper_2603_06588_b200 import binding

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hook_attn.h")
I32 = torch.int32


@pytest.fixture(scope="module")
def compiled():
    binding.load_library()
    return binding._compiled


@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


def test_every_call_of_the_header_is_exported():
    declared = re.findall(r"^\w[\w \*]*?\b(hook_\w+)\(", open(HEADER).read(), flags=re.M)
    assert sorted(declared) == sorted(binding.EXPORTS)
    lib = binding.load_library()
    assert all(hasattr(lib, name) for name in declared)
    assert set(binding._AROUND) <= set(binding.EXPORTS)


def _refused(call, *args):
    """Refused by the checks: the address of the entry point, 0, is never called.  A stream is given, so no device is asked for it."""
    with pytest.raises(AssertionError) as e:
        call(0, 0, 0, 0, *args)
    return str(e.value)


NAMES = ("rope_append", "adjust_logits", "cache_fork", "cache_extend", "cache_free", "cache_compact", "cache_copy_pages")
COUNTS = (16, 14, 6, 6, 6, 4, 4)


@pytest.mark.parametrize("name,count", list(zip(NAMES, COUNTS)))
def test_number_of_arguments(compiled, name, count):
    assert "number" in _refused(getattr(compiled, name), *[None] * (count + 1))
    assert "number" in _refused(getattr(compiled, name), *[None] * (count - 1))


@pytest.mark.parametrize("name,count", list(zip(NAMES, COUNTS))[:6])
@pytest.mark.parametrize("thing", [None, 7, "q", [torch.zeros(2)], torch.zeros(1, dtype=I32), torch.zeros((2, 3, 4))])
def test_first_argument(compiled, name, count, thing):
    """Nothing, no tensor, a tensor on the CPU."""
    _refused(getattr(compiled, name), thing, *[None] * (count - 1))


@pytest.mark.parametrize("caches", [[torch.zeros(1)], [(torch.zeros(1),)], [(None, None)], [(torch.zeros(1), torch.zeros(1))], ["kv"]])
def test_caches(compiled, caches):
    _refused(compiled.cache_copy_pages, caches, torch.zeros((1, 2), dtype=I32), None, None)


def test_caches_not_a_list(compiled):
    with pytest.raises(TypeError):
        compiled.cache_copy_pages(0, 0, 0, 0, 5, None, None, None)


@pytest.mark.parametrize("at", range(4))
def test_integers(compiled, at):
    """The four integers in front are integers."""
    head = [0, 0, 0, 0]
    head[at] = "x"
    args = [torch.zeros((1, 1), dtype=I32), None, None, None]
    with pytest.raises((TypeError, AssertionError)):
        compiled.cache_compact(*head, *args)


@pytest.mark.gpu
def test_gpu_refusals(eng):
    """On the device, one mistake each; the tensors come out as they went in."""
    t = lambda *shape, dtype=I32: torch.zeros(shape, dtype=dtype, device="cuda")
    pool = dict(block_table=t(2, 3), seq_lens=t(2), page_refs=t(8))
    for wrong in (dict(block_table=t(2, 3, dtype=torch.int64)), dict(block_table=t(2, 6)[:, ::2]), dict(seq_lens=t(3)), dict(seq_lens=t(2).cpu()),
                  dict(page_refs=t(8, 1)), dict(page_refs=t(16)[::2]), dict(status=t(1, dtype=torch.int64)), dict(status=t(0))):
        with pytest.raises(AssertionError):
            eng.hook_cache_compact(**{**pool, **wrong})
        with pytest.raises(AssertionError):
            eng.hook_cache_extend(**{**pool, **wrong}, new_rows=t(2))
    for wrong in (dict(new_rows=t(3)), dict(new_rows=t(2, dtype=torch.int64)), dict(new_rows=t(2), pairs=t(2, 3)), dict(new_rows=t(2), pairs=t(2, 4)[:, ::2])):
        with pytest.raises(AssertionError):
            eng.hook_cache_extend(**pool, **wrong)
    with pytest.raises(AssertionError):
        eng.hook_cache_fork(**pool, parents=t(2), children=t(1))
    with pytest.raises(AssertionError):
        eng.hook_cache_free(**pool, seqs=t(2), keep_lens=t(1))
    cache = t(4, 16, 2, 64, dtype=torch.bfloat16)
    for caches in ([(cache, cache.half())], [(cache, cache[:3])], [(cache, cache.cpu())], [(cache[..., ::2], cache[..., ::2])], [(cache, cache), (cache,)]):
        with pytest.raises(AssertionError):
            eng.hook_cache_copy_pages(caches, t(1, 2))
    for wrong in (dict(pairs=t(1, 3)), dict(pairs=t(1, 2, dtype=torch.int64)), dict(pairs=t(1, 4)[:, ::2]), dict(pairs=t(1, 2), num_pairs=t(2))):
        with pytest.raises(AssertionError):
            eng.hook_cache_copy_pages([(cache, cache)], **wrong)
    assert eng.hook_cache_copy_pages([], t(1, 2)) is None
    torch.cuda.synchronize()
    assert all(not x.any() for x in pool.values())


@pytest.mark.gpu
def test_results_are_the_tensors_given(eng):
    """What the caller gives for a result is what comes back, and a stream's number is taken as it is."""
    logits = torch.zeros((2, 40), device="cuda")
    out = torch.empty_like(logits)
    stream = torch.cuda.current_stream().cuda_stream
    assert eng.hook_adjust_logits(logits, out=out, stream=stream) is out and eng.hook_adjust_logits(logits) is logits
    pool = dict(block_table=torch.full((2, 3), -1, dtype=I32, device="cuda"), seq_lens=torch.zeros(2, dtype=I32, device="cuda"),
                page_refs=torch.zeros(8, dtype=I32, device="cuda"))
    pairs = torch.zeros((2, 2), dtype=I32, device="cuda")
    assert eng.hook_cache_extend(**pool, new_rows=torch.ones(2, dtype=I32, device="cuda"), pairs=pairs) is pairs
    assert pairs.tolist() == [[-1, -1]] * 2 and pool["seq_lens"].tolist() == [1, 1]
    table, refs, page_map, moves, count = eng.hook_cache_compact(**pool)
    assert table.shape == (2, 3) and refs.shape == (8,) and page_map.shape == (8,) and moves.shape == (4, 2) and count.shape == (1,)


@pytest.mark.gpu
def test_closed_handle(eng):
    mine = binding.HookAttn(0)
    mine.close()
    with pytest.raises(binding.HookAttnError) as e:
        mine.hook_adjust_logits(torch.zeros((2, 40), device="cuda"))
    assert e.value.code == binding.HOOK_ATTN_ERR_INVALID_ARG
