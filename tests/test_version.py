"""The package's version is the library's (CPU only)."""
import paper_2507_21433_amd
from paper_2507_21433_amd import binding as rc
from tests.test_abi import lib  # noqa: F401


def test_the_package_and_the_library_have_one_version(lib):
    major, minor, patch = (int(x) for x in paper_2507_21433_amd.__version__.split("."))
    assert rc.lib().rc_version() == major * 10000 + minor * 100 + patch
