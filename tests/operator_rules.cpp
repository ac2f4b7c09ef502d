// Rules of the norms and products that run on the host as well (test_operator_rules.py): one question per line of standard input.
#include <iostream>
#include <string>
#include <vector>

#include "rcd_elem.cuh"
#include "rcd_ring.h"

// A barrier that expects one arrival with the bytes of a copy: its phase ends when both are there.
struct Barrier {
    int pending = 1, phase = 0;
    bool bytes = false, copyUnderWay = false;
    bool twice = false;
    void order()
    {
        if (pending == 0) twice = true;
        --pending;
        bytes = copyUnderWay = true;
    }
    void arrive()
    {
        copyUnderWay = bytes = false;
        if (pending <= 0) { pending = 1; ++phase; }
    }
    bool done(uint32_t parity) const { return (uint32_t)(phase & 1) != parity; }
};

int main()
{
    std::string what;
    while (std::cin >> what) {
        if (what == "ring") {                              // slots, rows, then for each row: 0 its copy arrives, n: n waits later
            int stages, rows;
            std::cin >> stages >> rows;
            std::vector<int> late((size_t)rows);
            for (int &l : late) std::cin >> l;
            std::vector<Barrier> bars((size_t)stages);
            std::vector<int> due((size_t)stages, 0);
            auto order = [&](int row, int slot) {
                if (row >= rows) return;
                bars[slot].order();
                due[slot] = late[row];
            };
            for (int k = 0; k < stages; ++k) order(k, k);
            rcd::RingTurn at;
            int inTime = 0;
            for (int row = 0; row < rows; ++row) {
                for (int k = 0; k < stages; ++k)           // a wait's time passes
                    if (bars[k].copyUnderWay && due[k]-- == 0) bars[k].arrive();
                const bool came = bars[at.slot].done(at.parity);
                at.waited(came);
                inTime += came && at.may_order();
                if (at.may_order()) order(row + stages, at.slot);
                at.next(stages);
            }
            bool twice = false;
            for (const Barrier &b : bars) twice = twice || b.twice;
            std::cout << twice << " " << inTime << "\n";
        } else if (what == "meet") {                       // twice: address, rows, elements between rows, elements, bytes of one
            int64_t a[5], b[5];
            for (int64_t &x : a) std::cin >> x;
            for (int64_t &x : b) std::cin >> x;
            std::cout << rcd::ranges_meet((const void *)a[0], a[1], a[2], a[3], a[4], (const void *)b[0], b[1], b[2], b[3], b[4]) << "\n";
        } else {
            return 1;
        }
    }
    return 0;
}
