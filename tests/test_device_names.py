"""Names of the CUDA sources' types: all files share one namespace, so that two
types of one name would be one to the linker."""
import re

from test_device_source import FILES


def test_a_type_is_defined_once():
    where = {}
    for name, code in FILES.items():
        for kind in set(re.findall(r"^(?:struct|union|enum)\s+(?:class\s+)?(?:__align__\(\d+\)\s+)?(\w+)[^;{}<]*\{", code, re.M)):
            where.setdefault(kind, []).append(name)
    assert len(where) > 30 and {k: v for k, v in where.items() if len(v) > 1} == {}
