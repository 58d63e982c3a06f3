"""DEER draft-verify step on MI355X: thin Python binding over libdeer's C ABI."""
from .binding import DeerEngine, DeerError, Kv8Cache, load_library, LIB_PATH  # noqa: F401
