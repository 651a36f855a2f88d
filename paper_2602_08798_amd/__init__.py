"""MI355X-native server-side ciphertext x ciphertext attention path of CryptoGen.

All arithmetic runs in the HIP libraries (csrc/, built into libcryptogen_hip.so
and libcryptogen_requests.so) behind the C ABI declared in include/.  This package
only marshals arguments: PyTorch owns device memory and streams.  There is no CPU
fallback; loading raises if the evaluator has not been built, and making a
`Requests` if the second library has not.
"""
from .binding import Context, Library, load_library, to_device, to_host
from .serving import Requests

__all__ = ["Context", "Library", "Requests", "load_library", "to_device", "to_host"]
