// What the library's other translation units may ask of a store: its pool, its
// lock, its checks of caller pointers and its error message.
#pragma once

#include <cstdint>
#include <mutex>
#include <string>

#include "t2istore.h"

namespace t2i {

struct StoreInfo {
    uint64_t pool = 0;
    uint64_t total_pages = 0;
    uint64_t page_bytes = 0;
    int device = 0;
};

StoreInfo store_info(t2i_store* s);
std::mutex& store_mutex(t2i_store* s);
// (the rest with the lock held)
void store_set_error(t2i_store* s, std::string e);
// Device memory of the store's device that holds [p, p + n), outside the pool:
// a null-terminated reason where it is not. Consecutive calls between
// check_begin()s look an allocation up once.
void store_check_begin(t2i_store* s);
const char* store_check(t2i_store* s, const void* p, uint64_t n);
// Before and after a kernel launch: false where the testing hook fails it.
bool store_may_launch(t2i_store* s);
void store_launched(t2i_store* s);

}  // namespace t2i
