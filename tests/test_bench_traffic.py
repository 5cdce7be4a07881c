"""The stored traffic record of bench.py applies to the committed loop sources (CPU):
a change of one of them needs the record taken again, and what the loops do not use
belongs in a file of its own."""
import json

import bench


def test_the_record_applies():
    text = open(bench.TRAFFIC_FILE).read()
    entries = json.loads(text.split("```json", 1)[1].split("```", 1)[0])["entries"]
    assert entries
    for name, e in entries.items():
        assert bench.recorded_traffic(*name.split("/", 1)) == e["bytes_per_launch"], name
