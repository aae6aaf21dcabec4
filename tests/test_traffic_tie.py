"""What the stored traffic of contractions is tied to, besides their sources: the part of the header that they are declared by."""
import json

import pytest

from paper_2311_09549_amd import traffic


def test_header_without_attention(tmp_path):
    text = open(traffic.HEADER).read()
    digest = traffic.header_digest()
    def of(changed):
        path = tmp_path / "changed.h"
        path.write_text(changed)
        return traffic.header_digest(str(path))
    assert of(text) == digest
    for change in (("SC_ERR_ALLOC", "SC_ERR_ALLOC_"), ("typedef enum { SC_F32 = 0", "typedef enum { SC_F32 = 7"), ("sc_status sc_plan_destroy", "int sc_plan_destroy")):
        assert text.count(change[0]) >= 1 and of(text.replace(*change)) != digest
    assert of(text.replace("int32_t kv_heads;", "int64_t kv_heads;")) == digest       # attention's
    with pytest.raises(ValueError):
        of(text.replace(traffic.ATTENTION_DECLARATIONS, ""))


def test_stored_traffic_is_of_the_present_sources(tmp_path):
    with open(traffic.DEFAULT_PATH) as f:
        record = json.load(f)
    assert record["entries"]
    for key, entry in record["entries"].items():
        assert traffic.lookup(key) == entry
        for field in ("source_sha256", "header_sha256"):
            path = tmp_path / "traffic.json"
            path.write_text(json.dumps({"entries": {key: dict(entry, **{field: "0" * 64})}}))
            assert traffic.lookup(key, str(path)) is None
        path.write_text(json.dumps({"entries": {key: {k: v for k, v in entry.items() if k != "header_sha256"}}}))
        assert traffic.lookup(key, str(path)) is None
