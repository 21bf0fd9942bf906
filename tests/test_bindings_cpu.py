"""The binding's names: the types of the C arguments stay what they are when
tensors' types are checked (no GPU needed)."""
import ctypes


def test_argument_types_survive_tensor_checks(salt_lib):
    before = {n: getattr(salt_lib, n) for n in ("_vp", "_i32", "_i64", "_f32")}
    salt_lib._load_types()
    assert {n: getattr(salt_lib, n) for n in before} == before
    assert issubclass(salt_lib._i32, ctypes._SimpleCData) and ctypes.sizeof(salt_lib._i32 * 3) == 12
