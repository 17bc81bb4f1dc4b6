"""What decode over shared prefixes decides on the host, on the CPU: whether a launch could have a group whose prefix goes through shared
memory, and the workspace that goes by it."""
import ctypes

import pytest

import paper_2502_11880_amd as B

KEYS = (1024, 6016, 20000, 65536, 1 << 20)


def _may(columns, keys, kv_heads, dim, f32, three_parts):
    fn = B.lib()["_ZN6bitnet23attn_shared_may_be_wideElliibb"]
    fn.restype, fn.argtypes = ctypes.c_bool, [ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_bool, ctypes.c_bool]
    return fn(columns, keys, kv_heads, dim, f32, three_parts)


@pytest.mark.parametrize("f32,three_parts", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("dim", [4, 64, 80, 128, 132, 256])
@pytest.mark.parametrize("kv_heads", [1, 8, 32])
def test_other_sequences_never_keep_a_group_from_shared_memory(kv_heads, dim, f32, three_parts):
    """A launch may have any group of up to its own columns: what is worth it for one of them stays so beside others."""
    for keys in KEYS:
        may = [_may(c, keys, kv_heads, dim, f32, three_parts) for c in range(1, 2050)]
        first = may.index(True) if True in may else len(may)
        assert all(may[first:]), (keys, first + 1, may.index(False, first) + 1)
        assert not any(may[:64]), "up to 64 columns go through registers"


def test_some_prefixes_go_through_shared_memory():
    """Thousands of columns behind a long prefix do, in every type."""
    for dim in (64, 128, 256):
        for f32, three_parts in ((False, False), (True, False), (True, True)):
            assert _may(2048, 1 << 20, 8, dim, f32, three_parts)


@pytest.mark.parametrize("dim", [64, 100, 128, 256])
def test_workspace_grows_with_the_batch(dim):
    for heads, kv_heads in ((32, 8), (32, 32), (64, 1)):
        for max_pages in (10, 100, 1024, 4096):
            sizes = [B.bitnet_attn_decode_shared_workspace_bytes(n, heads, kv_heads, dim, 64, max_pages) for n in range(1, 1100)]
            assert sizes == sorted(sizes)


@pytest.mark.parametrize("f32,three_parts", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("dim", [132, 160, 192, 224, 252])
def test_heads_between_128_and_256_go_through_registers(dim, f32, three_parts):
    """Measured there 1.2 to 2.4 times as fast, at 128 to 512 columns of 1 to 32 kv heads behind 6016 and 32768 keys."""
    assert not any(_may(c, keys, kv_heads, dim, f32, three_parts) for c in (128, 256, 512, 2048) for keys in KEYS for kv_heads in (1, 8, 32))


@pytest.mark.parametrize("dim,least,most,wide", [(64, 4, 18, 36), (128, 9, 18, 70), (256, 17, 35, 137)])
def test_workspace_has_the_stated_size(dim, least, most, wide):
    """In MB: what the header says, with and without prefixes that could go through shared memory, and the records of whole rows."""
    for heads, kv_heads in ((1, 1), (32, 8), (32, 32), (64, 1), (96, 12)):
        for n in (1, 7, 64, 1024, 5000):
            for max_pages in (1, 20, 1024, 1 << 18):
                got = B.bitnet_attn_decode_shared_workspace_bytes(n, heads, kv_heads, dim, 64, max_pages) / 1e6
                twice = 2 * min(n, 1024) * heads * (dim + 4) * 4 / 1e6
                assert least - 0.5 < got - twice <= most or least + wide - 1 < got - twice <= most + wide, (heads, kv_heads, n, max_pages)


# Sent both ways on the device: where the difference was more than 12% of the time, the rule takes the faster one.
@pytest.mark.parametrize("dim,f32,three_parts,columns,kv_heads,keys,shared", [
    (64, 0, 0, 256, 1, 32768, True), (64, 0, 0, 512, 8, 1024, False), (64, 0, 0, 80, 1, 6016, False), (64, 0, 0, 256, 32, 6016, True),
    (32, 0, 0, 512, 32, 6016, True), (64, 1, 0, 80, 8, 6016, False), (64, 1, 0, 256, 8, 32768, True), (64, 1, 0, 512, 8, 1024, False),
    (64, 1, 1, 80, 8, 6016, False), (64, 1, 1, 128, 32, 32768, True), (64, 1, 1, 256, 32, 1024, False), (48, 1, 1, 512, 32, 6016, True),
    (128, 0, 0, 80, 8, 32768, True), (128, 0, 0, 256, 1, 32768, False), (112, 0, 0, 512, 8, 6016, True), (80, 0, 0, 128, 8, 6016, False),
    (128, 1, 0, 80, 1, 32768, False), (128, 1, 0, 128, 32, 6016, True), (80, 1, 0, 128, 8, 32768, True), (100, 1, 0, 80, 8, 16000, False),
    (128, 1, 1, 128, 8, 32768, True), (128, 1, 1, 80, 32, 6016, False), (100, 1, 1, 512, 1, 32768, False), (112, 1, 1, 512, 32, 6016, True),
    (256, 0, 0, 80, 8, 6016, False), (256, 0, 0, 80, 8, 32768, True), (256, 0, 0, 512, 32, 1024, True), (256, 0, 0, 128, 1, 32768, False),
    (256, 1, 0, 80, 8, 32768, False), (256, 1, 0, 512, 32, 6016, True), (256, 1, 0, 256, 8, 32768, True), (256, 1, 0, 256, 32, 1024, False),
    (256, 1, 1, 80, 32, 32768, False), (256, 1, 1, 128, 32, 32768, True), (256, 1, 1, 512, 8, 6016, False), (256, 1, 1, 512, 8, 32768, True)])
def test_the_rule_takes_the_faster_way(dim, f32, three_parts, columns, kv_heads, keys, shared):
    assert _may(columns, keys, kv_heads, dim, bool(f32), bool(three_parts)) is shared
