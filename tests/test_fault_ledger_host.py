"""A fault of the attention kernels is told to every host thread and stream that asks, once each (no device work)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <stdio.h>
#include <thread>
#include "faults.h"
static thread_local FaultLedger ledger;
int main() {
    int a, b;
    auto ask = [&](int device, void *stream, unsigned count) { putchar(ledger.news(device, stream, count) ? '1' : '0'); };
    ask(0, &a, 0);                       // nothing yet
    ask(0, &a, 1), ask(0, &a, 1);        // a fault: told once
    ask(0, &b, 1), ask(0, &b, 1);        // another stream is told too
    ask(1, &a, 0), ask(1, &a, 2);        // another device counts for itself
    ask(0, &b, 5), ask(0, &a, 5);        // more faults: both again
    std::thread([&] { ask(0, &a, 5), ask(0, &a, 5); }).join();   // another thread on the same stream
    ask(0, &a, 5);
}
'''


def test_every_caller_is_told_once(tmp_path):
    (tmp_path / "ledger.cpp").write_text(SOURCE)
    exe = tmp_path / "ledger"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-pthread", "-I", os.path.join(ROOT, "paper_2603_01501_b200", "csrc"), "-o",
                    str(exe), str(tmp_path / "ledger.cpp")], check=True)
    told = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.strip()
    assert told == "0" "10" "10" "01" "11" "10" "0"

