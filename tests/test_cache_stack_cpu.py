"""CacheStack's descriptors are checked at every call, on tensors of the CPU that are let pass for the GPU's: a tensor
that was resized, transposed or given other memory in place is refused before the library is called, in whichever layer
it is."""
import pytest
import torch

from paper_2510_09883_amd import delta as D
from paper_2510_09883_amd import drafts as T
from paper_2510_09883_amd import extend as E

LAYERS = 5


def _dev(name, t, dtype=None, shape=None, at_least=None):
    """delta._dev, but for where the tensor is."""
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if shape is not None and (t.dim() != len(shape) or any(w not in (None, x) for w, x in zip(shape, t.shape))):
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    return t


@pytest.fixture
def calls(monkeypatch):
    """What the library is called with."""
    got = []
    for module in (D, E, T):
        monkeypatch.setattr(module, "_dev", _dev)
    monkeypatch.setattr(T, "_stream_of", lambda *a: None)
    monkeypatch.setattr(D._lib, "delta_cache_compact", lambda *a: got.append(a) or D.DELTA_OK)
    return got


def stack_of(e4m3, heads=2, own_tables=False):
    kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    lens, table = torch.tensor([40, 60], dtype=torch.int32), torch.zeros((2, 4), dtype=torch.int32)
    kvs = []
    for _ in range(LAYERS):
        k, v = (torch.zeros((9, heads, 16, 64), dtype=torch.uint8 if e4m3 else torch.int16).view(kind) for _ in range(2))
        scale = dict(k_scale=torch.ones(heads), v_scale=torch.ones(heads)) if e4m3 else {}
        kvs.append(D.make_kv(k, v, table.clone() if own_tables else table, lens, **scale))
    return T.CacheStack(D.make_shape(2, 2 * heads, heads, 64, 4, 60), kvs)


def compact(stack):
    path = torch.zeros((2, 3), dtype=torch.int32)
    T.delta_cache_compact(stack, 6, torch.tensor([0, 3, 6], dtype=torch.int32), path, path[:, 0].contiguous())


def _other_memory(t):
    t.data = t.clone()


CHANGES = [(2, lambda t: t.resize_(2, 3), "^page_table: expected shape"), (3, lambda t: t.resize_(1), "^seq_lens: expected shape"),
           (0, lambda t: t.resize_(9, 2, 8, 64), "^k_cache: expected shape"),
           (1, lambda t: t.resize_(9, 2, 32, 32), "^v_cache: expected shape"),       # (as many elements)
           (1, lambda t: t.transpose_(2, 3), "^v_cache"), (0, lambda t: t.transpose_(1, 2), "^k_cache: must be contiguous"),
           (0, _other_memory, "^k_cache: its memory"), (2, _other_memory, "^page_table: its memory"),
           (3, lambda t: t.set_(torch.zeros(2, dtype=torch.int32)), "^seq_lens: its memory"),
           (1, lambda t: t.resize_(400, 2, 16, 64), "^v_cache: its memory")]      # (more than it has room for)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("layer", [0, LAYERS - 1])
@pytest.mark.parametrize("which,change,match", CHANGES)
def test_a_tensor_changed_in_place_is_refused(calls, which, change, match, layer, e4m3):
    stack = stack_of(e4m3, 16 if "contiguous" in match else 2, own_tables=True)
    compact(stack)
    assert len(calls) == 1
    t = stack.layers[layer]._tensors[which]
    kept = t.data   # (the memory that a call would write)
    change(t)
    for _ in range(2):
        with pytest.raises(ValueError, match=match):
            compact(stack)
    assert len(calls) == 1 and kept.numel()


def test_a_shape_changed_in_place_is_refused(calls):
    for name, value in (("batch", 3), ("n_kv_heads", 1), ("head_dim", 128), ("max_pages_per_seq", 3)):
        stack = stack_of(False)
        compact(stack)
        setattr(stack.shape, name, value)
        with pytest.raises(ValueError, match="expected shape"):
            compact(stack)
    assert len(calls) == 4


def test_what_has_not_changed_passes(calls):
    """Contents written in place, and a cache of fewer pages in the same memory, as any other call takes it."""
    stack = stack_of(True)
    compact(stack)
    for x in stack.layers[1]._tensors[:4]:
        x.zero_() if x.dtype == torch.int32 else x.view(torch.uint8).fill_(3)
    compact(stack)
    stack.layers[2]._tensors[0].resize_(8, 2, 16, 64)
    compact(stack)
    assert len(calls) == 3
    by_hand = [D.delta_kv_t(0x1000 * i, 0x800 + 0x1000 * i, 0x1000, 0x1000, 0, 0, None, None) for i in (1, 2)]
    compact(T.CacheStack(stack.shape, by_hand))    # (raw addresses: nothing to check)
    assert len(calls) == 4
