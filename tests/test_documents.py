"""The documents at the top: what they point to is there, and every measured case stands in one of their tables."""
import re
from pathlib import Path

import pytest

from perf import more_operators, operators

ROOT = Path(__file__).resolve().parent.parent
DOCUMENTS = {p.name: p.read_text() for p in ROOT.glob("*.md")}


def headings(text):
    return set(re.findall(r"^#+ (\d+)\.", text, re.M))


@pytest.mark.parametrize("name", sorted(n for n, t in DOCUMENTS.items() if len(headings(t)) > 4 and "**Measured**" in t))
def test_sections_that_a_document_points_to_are_there(name):
    own = DOCUMENTS[name]
    missing = set(re.findall(r"§(\d+)", own)) - headings(own)
    assert not missing, f"{name}: no section {sorted(missing)}"


def test_sections_of_other_documents_are_there():
    for name, text in DOCUMENTS.items():
        for other, section in re.findall(r"`(\w+\.md)` §(\d+)", text):
            if other in DOCUMENTS and headings(DOCUMENTS[other]):
                assert section in headings(DOCUMENTS[other]), f"{name}: {other} has no section {section}"


@pytest.mark.parametrize("module", [operators, more_operators], ids=["products", "norms"])
def test_every_measured_case_stands_in_a_table_and_among_what_is_left(module):
    """Its floor, the plain form's time and the kernel's in one row; and by name where the reasons stand for what was left as it is."""
    for case in module.listed():
        name = case["name"]
        rows = [r for t in DOCUMENTS.values() for r in re.findall(rf"^\| `{name}` \|.*$", t, re.M)]
        assert len(rows) == 1 and rows[0].count("|") == 7, f"{name}: {rows}"
        assert any(f"`{name}`" in part for t in DOCUMENTS.values() for part in re.findall(r"\*\*Left as it is[^#]*", t)), f"{name}: no reason"
