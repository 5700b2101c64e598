"""Host-side checks of the operators over a caller's paged cache (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import cache_helpers as H
from paper_2511_08923_b200 import Tidar, TidarError, binding, kv4_page_bytes


def test_page_bytes():
    assert kv4_page_bytes(64) == 64 * (32 + 8) and kv4_page_bytes(128) == 64 * (64 + 16)
    for hd in (0, 32, 96, 256, -64):
        with pytest.raises(TidarError):
            kv4_page_bytes(hd)
    assert binding.load().tidar_kv4_page_bytes(64, None) == -1


def test_calls_without_a_context_are_refused():
    lib = binding.load()
    assert lib.tidar_page_map(None, *[None] * 3, 1, None, 0, None, None, 1, None, None, None, 0, None) == -1
    assert lib.tidar_kv4_store(None, None, 8, None, 8, None, 0, None, None, 1) == -1
    assert lib.tidar_kv4_load(None, None, None, 1, None, 0, None, 8, None, 8) == -1
    assert lib.tidar_attention_kv4(None, None) == -1 and lib.tidar_attention_window(None, None) == -1


def test_the_binding_refuses_tensors_of_another_device_type_or_shape():
    t = Tidar.__new__(Tidar)
    t._index = 0
    for x in (torch.zeros(3), torch.zeros(3, dtype=torch.int32), None, [1, 2]):
        with pytest.raises(ValueError):
            t._tensor("x", x, torch.float32, (3,))
    t._index = -1                                        # (where a CPU tensor says it is, so that the other checks are reached)
    x = torch.zeros(4, 6, 8)
    assert t._tensor("x", x, torch.float32, (4, 6, 8)) == x.data_ptr()
    assert t._rows("x", x[:, 1:3], torch.float32, (4, 2, 8)) == (x.data_ptr() + 32, 48)
    assert t._rows("x", x[:1, 1:3], torch.float32, (1, 2, 8)) == (x.data_ptr() + 32, 16) and t._rows("x", x[:, 2:3], torch.float32, (4, 1, 8))[1] == 48
    assert t._rows("x", x[:0], torch.float32, (0, 6, 8))[1] == 48
    for bad, dtype, shape in ((x[:, :, ::2], torch.float32, (4, 6, 4)), (x[:, ::2], torch.float32, (4, 3, 8)), (x.transpose(0, 1), torch.float32, (6, 4, 8)), (x.half(), torch.float32, (4, 6, 8)),
                              (x, torch.float32, (4, 6, 9)), (x[:1].expand(4, 6, 8), torch.float32, (4, 6, 8)), (x[0], torch.float32, (4, 6, 8)), (None, torch.float32, (1, 1, 1))):
        with pytest.raises(ValueError):
            t._rows("x", bad, dtype, shape)
    with pytest.raises(ValueError):
        t._tensor("x", x[:, 1:3], torch.float32, (4, 2, 8))
    with pytest.raises(ValueError):
        Tidar._length("x", torch.zeros(3), 1)
    with pytest.raises(ValueError):
        Tidar._length("x", [1], 0)


def test_argument_struct_is_laid_out_as_in_c(tmp_path):
    """Offsets of tidar_attention_args as the C compiler has them."""
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in binding.tidar_attention_args._fields_]
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "o.c"
    src.write_text('#include <stdio.h>\n#include "tidar.h"\nint main(void) {\n' + "".join(f'printf("%zu ", offsetof(tidar_attention_args, {n}));\n' for n in names) +
                   'printf("%zu", sizeof(tidar_attention_args)); return 0; }\n')
    subprocess.run([cc, "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "o")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "o")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(binding.tidar_attention_args, n).offset for n in names] + [C.sizeof(binding.tidar_attention_args)]


def test_the_plain_statement_of_4_bit_rows():
    """Codes come back as the values that the definition names, and those are within a step of what was stored."""
    rng = np.random.default_rng(1)
    x = H.bf16_round(rng.standard_normal((3, 64, 128)) * 3)
    c, s, b = H.quantise(x)
    assert c.min() >= 0 and c.max() <= 15
    y = H.values(c, s, b)
    assert (np.abs(y - x) <= np.repeat(s, 32, -1) * 0.75 + 2.0 ** -8 * np.abs(x)).all()
    rec = H.records(x)
    assert rec.shape == (3, kv4_page_bytes(128))
    word = rec[0, :4].astype(np.uint32)
    word = word[0] | word[1] << 8 | word[2] << 16 | word[3] << 24
    assert [int(word >> (4 * (d // 2) + 16 * (d % 2)) & 15) for d in range(8)] == c[0, 0, :8].tolist()
    # how readers get from codes to values: 16 + c is the bf16 number with the code in its upper mantissa bits
    for code in range(16):
        assert np.array([0x4180 | code << 3], dtype=np.uint32).__lshift__(16).view(np.float32)[0] == 16 + code


def test_visibility_by_cases():
    v = H.visible(10, 2, True, 4, 3, 12)
    assert np.nonzero(v[0])[0].tolist() == [0, 1, 2, 7, 8, 9, 10]           # causal slot 0, position 10
    assert np.nonzero(v[1])[0].tolist() == [0, 1, 2, 8, 9, 10, 11]
    assert np.nonzero(v[2])[0].tolist() == [0, 1, 2, 8, 9, 10]              # block 0, slot 0: position 11
    assert np.nonzero(v[5])[0].tolist() == [0, 1, 2, 10, 11]                # block 1, slot 1: position 13
    assert H.visible(10, 2, True, 0, 0, 12)[5].sum() == 12


def _recorder(hq=4, hkv=2, hd=64):
    """A binding object whose library calls are recorded instead of made; CPU (and meta) tensors count as on its device."""
    from types import SimpleNamespace
    t = Tidar.__new__(Tidar)
    t._index, t.shape, t.lib, t.ctx, t.calls = -1, SimpleNamespace(n_q_heads=hq, n_kv_heads=hkv, head_dim=hd), binding.load(), None, []
    t._on_device = lambda entry, *args: t.calls.append(args)
    return t


def test_the_binding_refuses_numbers_that_the_library_cannot_hold():
    """Integers are 32 bits in the library: 2^32 + 5 would arrive there as 5."""
    t, bf = _recorder(), torch.bfloat16
    q, out, n, table = torch.zeros(1, 4, 64, dtype=bf), torch.zeros(1, 256, dtype=bf), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 3, dtype=torch.int32)
    pools = {t.attention_kv4: torch.zeros(3, 2, kv4_page_bytes(64), dtype=torch.uint8), t.attention_window: torch.zeros(3, 2, 64, 64, dtype=bf)}
    for call, pool in pools.items():
        for good in (dict(window=0), dict(window=2 ** 31 - 1, sinks=2 ** 31 - 1)):
            t.calls.clear()
            call(q, pool, pool, table, n, None, None, out, 1, 1, **good)
            args = t.calls[0][0]._obj
            assert args.window == good["window"] and args.sinks == good.get("sinks", 0)
        t.calls.clear()
        for bad in (dict(window=2 ** 31), dict(window=2 ** 32 + 5), dict(window=-2 ** 31 - 1), dict(window=9, sinks=2 ** 32), dict(window=9, sinks=-2 ** 32)):
            with pytest.raises(ValueError):
                call(q, pool, pool, table, n, None, None, out, 1, 1, **bad)
    many, one = 2 ** 32 + 5, lambda k: torch.zeros(k, dtype=torch.int32)
    meta = lambda *s, dtype=torch.int32: torch.empty(*s, dtype=dtype, device="meta")
    for free, slots, wide in ((one(4), meta(many), table), (meta(many), one(4), table), (one(4), one(4), meta(1, many))):
        with pytest.raises(ValueError):
            t.page_map(n, n, n, free, wide, one(1), one(2), slots, one(3))
    rows, pool = meta(many, 2, 64, dtype=bf), meta(3, 2, kv4_page_bytes(64), dtype=torch.uint8)
    with pytest.raises(ValueError):
        t.kv4_store(rows, rows, meta(many), pool, pool)
    with pytest.raises(ValueError):
        t.kv4_load(pool, pool, meta(many), rows, rows)
    pool = meta(many, 2, kv4_page_bytes(64), dtype=torch.uint8)
    with pytest.raises(ValueError):
        t.kv4_store(meta(7, 2, 64, dtype=bf), meta(7, 2, 64, dtype=bf), one(7), pool, pool)
    assert not t.calls
    t.page_map(n, n, n, one(4), table, one(1), one(2), one(4), one(3))
    assert len(t.calls) == 1
